// tv_attend_tile.cu -- attention over the 4-bit key/value cache for many query rows per
// key/value head (sm_103a): large trees and pieces of prompts, on the 5th-generation tensor
// cores.  Mathematics, rounding and the cut into pieces are those of tv_attend.cu.
//
// One persistent CTA per SM, two tiles of 128 rows at a time:
//   warps 0-3, 4-7    softmax of tile 0 and 1, one row per thread: scores from tensor
//                     memory, weights back into it as fp16, over the scores' first half
//   warps 8-11        widen 128 tokens' keys to fp16 in shared memory (a token per thread,
//                     its codes loaded a step ahead), two stages
//   warps 12-15       the same for values
//   warp 16           the products: S = Q K^T (both from shared memory) and O += P V (P
//                     from tensor memory), S and O of both tiles in tensor memory
//   warp 17           the CTA's pieces, in a ring that the others read
//   warps 18, 19      zeros in the rows behind the requests' last
// (the registers that these four leave go to the softmax).
// The two tiles take turns: while one's scores become weights, the tensor cores work on the
// other.  Where an item has 128 rows or fewer both tiles are the same rows and take
// alternate steps, and their sums are joined at the end.
// Steps go from the last tokens to the first, so that a row's path to the root is walked once,
// and the tree's tokens, which rows see in part, come first.
//
// A product that overwrites a tile's scores is issued after the one that reads its weights,
// by the same thread: the tensor cores take them in that order.  Every wait is bounded; one that
// gives up raises the timeout status, and the loops go on to their end.
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/tv.h"
#include "tv_attend.cuh"
#include "tv_launch.h"
#include "tv_umma.cuh"

namespace tvk {
namespace attend {

using namespace gemm;

constexpr int kTile = 128;
constexpr int kSoftmaxWarps = 8;
constexpr int kWidenWarps = 8;                   // four for keys, four for values
constexpr int kMmaWarp = kSoftmaxWarps + kWidenWarps;
constexpr int kTileThreads = 32 * (kMmaWarp + 4);
// registers per thread after the split
constexpr int kRegsSoftmax = 136, kRegsWiden = 72, kRegsMma = 64, kRegsLaunch = 96;
static_assert(32 * (kSoftmaxWarps * kRegsSoftmax + kWidenWarps * kRegsWiden + 4 * kRegsMma) <=
                  kTileThreads * kRegsLaunch,
              "the warpgroups' registers fit what the block was launched with");
constexpr int kStages = 2;
constexpr int kOkSlots = 4;
constexpr uint32_t kHalfBytes = kTile * 128;     // 64 columns (128 bytes) of a tile's rows
constexpr int kJoinParts = 8;                    // blocks that join one item's rows

// An item that begins in a CTA and goes on in later ones, up to `last`; b < 0: there is none.
struct Split {
  int b, head, m0, last;
};

// A piece as the warps take it; more = 0: there is none.
struct Work {
  int more, b, head, m0, s0, s1, steps, tokens, len, rows;
  __device__ __forceinline__ bool whole() const { return s0 == 0 && s1 == steps; }
};
constexpr int kWorkSlots = 4;
constexpr int kTakers = kSoftmaxWarps + kWidenWarps + 1;

struct TileShared {
  uint64_t given[kWorkSlots], taken[kWorkSlots];
  Work work[kWorkSlots];
  int softmax_more;
  uint64_t kfull[kStages], kempty[kStages], vfull[kStages], vempty[kStages];
  uint64_t sfull[2], pfull[2], ofull[2], qfull;
  uint32_t tmem;
  // tokens of a step that exist and have a page; a slot is used again four steps later, when
  // both softmaxes are done with it
  uint4 ok[kOkSlots];
  float m[2][kTile], l[2][kTile];
  Schedule plan;
  int32_t parents[1024];
};

template <int kRegs>
__device__ __forceinline__ void regs_fewer() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void regs_more() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}

__device__ __forceinline__ void wait_on(uint64_t* bar, uint32_t parity, uint32_t& bad) {
  if (!mbar_try_wait(bar, parity) && !bad) bad = mbar_wait(bar, parity) ? 0u : 1u;
}

// The n-th piece.  Whether there is one is only one thread's or one warp's to say: after a
// wait that gave up others may see something else.
__device__ __forceinline__ const Work* take(TileShared& sh, uint32_t n, uint32_t& bad) {
  wait_on(&sh.given[n % kWorkSlots], (n / kWorkSlots) & 1, bad);
  const Work* const w = &sh.work[n % kWorkSlots];
  return __all_sync(0xffffffffu, !bad && w->more) ? w : nullptr;
}
__device__ __forceinline__ void give_back(TileShared& sh, uint32_t n) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.taken[n % kWorkSlots]);
}

// Descriptor of an operand whose rows are 128 bytes (with the 128-byte swizzle) and whose
// columns are the other dimension than that of the sum: 8 rows of the sum's dimension after
// 1024 bytes, the next 64 columns after kHalfBytes.
__device__ __forceinline__ uint64_t column_desc(const void* p) {
  const uint64_t addr = smem_u32(p);
  return ((addr >> 4) & 0x3FFFull) | ((uint64_t)(kHalfBytes >> 4) << 16) |
         ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor of kind::f16: fp32 accumulator (bits 4-5 = 1), fp16 A and B (0), B by
// columns (bit 16), N >> 3 in bits 17-22, M >> 4 in bits 24-28.
__device__ __forceinline__ constexpr uint32_t f16_desc(int m, int n, bool by_columns) {
  return (1u << 4) | ((by_columns ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                 "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
      "%28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_stored() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void async_visible() {      // shared memory written, for the products
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void softmax_barrier() {    // both softmaxes' threads
  asm volatile("bar.sync 1, %0;" ::"n"(32 * kSoftmaxWarps) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c,
                                       uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c),
               "r"(d)
               : "memory");
}
// Where 16-byte piece x (8 columns) of row r of a tile is.
__device__ __forceinline__ uint32_t piece_at(uint32_t base, int r, int x) {
  return base + (uint32_t)(x >> 3) * kHalfBytes + (uint32_t)r * 128u +
         (uint32_t)(((x & 7) ^ (r & 7)) << 4);
}

// The codes and scales of a token's keys or values.
template <int D>
struct Token {
  uint4 code[D / 32];
  uint32_t scale[D / 32];
  bool there;
  __device__ __forceinline__ void load(const AttendArgs& a, const Work& p, int pos, int side) {
    const int page = pos < p.tokens ? page_of(a.c, a.t, p.b, pos) : -1;
    there = page >= 0;
    if (there) {
      const uint8_t* const block = block_of(a.c, a.layer, page, p.head, side);
      const int slot = pos & (a.c.page_size - 1);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const size_t at = (size_t)c * a.c.page_size + slot;
        code[c] = __ldg(reinterpret_cast<const uint4*>(block + at * 16));
        scale[c] = __ldg(reinterpret_cast<const uint16_t*>(
            block + (size_t)a.c.page_size * D / 2 + at * 2));
      }
    } else {
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        code[c] = make_uint4(0, 0, 0, 0);
        scale[c] = 0;
      }
    }
  }
  __device__ __forceinline__ void widen_to(uint32_t base, int row) const {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const uint32_t s2 = decode_scales(scale[c]), lo = lo_lo(s2), hi = hi_hi(s2);
      const uint32_t w[4] = {code[c].x, code[c].y, code[c].z, code[c].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t h[4];
        decode8(w[i], h);
        const uint32_t s = i < 2 ? lo : hi;
        sts128(piece_at(base, row, 4 * c + i), mul2(h[0], s), mul2(h[1], s), mul2(h[2], s),
               mul2(h[3], s));
      }
    }
  }
};

__device__ __forceinline__ void hide(uint32_t (&c)[32], uint32_t see) {
#pragma unroll
  for (int y = 0; y < 32; ++y)
    if (!(see >> y & 1)) c[y] = 0xff800000u;
}
// The lowest n bits of a word that holds bits [at, at + 32).
__device__ __forceinline__ uint32_t low_bits(int n, int at) {
  const int k = n - at;
  return k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u;
}

// The scratch: two pieces of every CTA, their rows' (maximum, sum), the CTAs' split items.
__device__ __forceinline__ float2* stats_of(const AttendArgs& a, int D, int ctas) {
  return reinterpret_cast<float2*>(a.part + (size_t)2 * ctas * 2 * kTile * D);
}
__device__ __forceinline__ Split* splits_of(const AttendArgs& a, int D, int ctas) {
  return reinterpret_cast<Split*>(stats_of(a, D, ctas) + (size_t)2 * ctas * 2 * kTile);
}

template <int D>
__global__ void __launch_bounds__(kTileThreads, 1) tile_kernel(AttendArgs a, int split, int wide) {
  constexpr uint32_t kTileBytes = kTile * D * 2;
  extern __shared__ uint8_t smem_raw[];
  __shared__ TileShared sh;
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* const q_tiles = smem;                               // [2]
  uint8_t* const k_tiles = smem + 2 * kTileBytes;              // [kStages]
  uint8_t* const v_tiles = k_tiles + kStages * kTileBytes;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rows_of_item = split ? kTile : 2 * kTile;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.kfull[i], 4);
      mbar_init(&sh.kempty[i], 1);
      mbar_init(&sh.vfull[i], 4);
      mbar_init(&sh.vempty[i], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sh.sfull[x], 1);
      mbar_init(&sh.pfull[x], 4);
      mbar_init(&sh.ofull[x], 1);
    }
    mbar_init(&sh.qfull, kSoftmaxWarps);
    for (int i = 0; i < kWorkSlots; ++i) {
      mbar_init(&sh.given[i], 1);
      mbar_init(&sh.taken[i], kTakers);
    }
    fence_mbar_init();
  }
  if (warp == kMmaWarp) tmem_alloc<false>(&sh.tmem);
  Walker walker;
  const Shares shares = plan(a, sh.plan, rows_of_item, blockIdx.x, gridDim.x, walker);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  uint32_t bad = 0, taken = 0;                   // pieces so far

  if (warp >= kMmaWarp) {
    // ---- products ----
    regs_fewer<kRegsMma>();
    if (warp == kMmaWarp) {
      const uint64_t qd[2] = {smem_desc(q_tiles), smem_desc(q_tiles + (split ? 0 : kTileBytes))};
      const uint64_t kd = smem_desc(k_tiles), vd = column_desc(v_tiles);
      uint32_t steps_done = 0, pcount[2] = {0, 0};
      for (; const Work* const w = take(sh, taken, bad); ++taken) {
        const int n = w->s1 - w->s0, ops = split ? n : 2 * n;
        give_back(sh, taken);
        wait_on(&sh.qfull, taken & 1, bad);
        tc_fence_after();
        auto scores = [&](int i, int x) {
          const uint32_t s = steps_done + (split ? i : i >> 1), stage = s % kStages;
          if (split || x == 0) {
            wait_on(&sh.kfull[stage], (s / kStages) & 1, bad);
            tc_fence_after();
          }
          if (elect_one()) {
  #pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint32_t off = (uint32_t)((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
              mma_ss(tmem + x * kTile, qd[x] + off, kd + stage * (kTileBytes >> 4) + off,
                     f16_desc(kTile, kTile, false), k > 0);
            }
            umma_commit<false>(&sh.sfull[x]);
            if (split || x == 1) umma_commit<false>(&sh.kempty[stage]);
          }
          __syncwarp();
        };
        auto values = [&](int i, int x) {
          const uint32_t s = steps_done + (split ? i : i >> 1), stage = s % kStages;
          if (split || x == 0) wait_on(&sh.vfull[stage], (s / kStages) & 1, bad);
          wait_on(&sh.pfull[x], pcount[x] & 1, bad);
          ++pcount[x];
          tc_fence_after();
          if (elect_one()) {
  #pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
              mma_ts(tmem + 2 * kTile + x * D, tmem + x * kTile + k * 8,
                     vd + stage * (kTileBytes >> 4) + k * (2048u >> 4), f16_desc(kTile, D, true),
                     i >= 2 || k > 0);
            umma_commit<false>(&sh.ofull[x]);
            if (split || x == 1) umma_commit<false>(&sh.vempty[stage]);
          }
          __syncwarp();
        };
        scores(0, 0);
        if (ops > 1) scores(1, 1);
        for (int i = 0; i < ops; i += 2) {
          values(i, 0);
          if (i + 2 < ops) scores(i + 2, 0);
          if (i + 1 < ops) {
            values(i + 1, 1);
            if (i + 3 < ops) scores(i + 3, 1);
          }
        }
        steps_done += (uint32_t)n;
      }
    } else if (warp == kMmaWarp + 1 && lane == 0) {
      // ---- pieces ----
      Piece p;
      Split split_item = {-1, 0, 0, 0};
      for (uint32_t n = 0;; ++n) {
        wait_on(&sh.taken[n % kWorkSlots], ((n / kWorkSlots) & 1) ^ 1, bad);
        Work w = {};
        if (!bad && walker.next(a, rows_of_item, p)) {
          w = Work{1, p.b, p.head, p.m0, p.s0, p.s1, p.steps, p.tokens, p.rq.len, p.rq.rows};
          if (p.s0 == 0 && p.s1 < p.steps)
            split_item = Split{p.b, p.head, p.m0, shares.owner(p.first + p.steps - 1)};
        }
        sh.work[n % kWorkSlots] = w;
        mbar_arrive(&sh.given[n % kWorkSlots]);
        if (!w.more) break;
      }
      splits_of(a, D, gridDim.x)[blockIdx.x] = split_item;
    } else if (warp > kMmaWarp + 1) {
      zero_rows(a, D, blockIdx.x * 2 + (warp & 1), gridDim.x * 2);
    }
  } else if (warp >= kSoftmaxWarps) {
    // ---- keys and values to fp16 ----
    regs_fewer<kRegsWiden>();
    const int side = warp >= kSoftmaxWarps + 4, row = tid & (kTile - 1);
    uint64_t* const full = side ? sh.vfull : sh.kfull;
    uint64_t* const empty = side ? sh.vempty : sh.kempty;
    const uint32_t base = smem_u32(side ? v_tiles : k_tiles);
    uint32_t s = 0;
    for (; const Work* const w = take(sh, taken, bad); ++taken) {
      const Work p = *w;
      Token<D> next;
      next.load(a, p, (p.s1 - 1) * kStep + row, side);
      for (int step = p.s1 - 1; step >= p.s0; --step, ++s) {
        const Token<D> now = next;
        if (step > p.s0) next.load(a, p, (step - 1) * kStep + row, side);
        const uint32_t stage = s % kStages;
        wait_on(&empty[stage], ((s / kStages) & 1) ^ 1, bad);
        now.widen_to(base + stage * kTileBytes, row);
        if (!side) {
          const uint32_t word = __ballot_sync(0xffffffffu, now.there);
          if (lane == 0) reinterpret_cast<uint32_t*>(&sh.ok[s % kOkSlots])[warp & 3] = word;
          if (!now.there && step * kStep + row < p.tokens)
            atomicOr(a.status, (uint32_t)TV_STATUS_BAD_PAGE);
        }
        async_visible();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[stage]);
      }
      give_back(sh, taken);
    }
  } else {
    // ---- softmax ----
    regs_more<kRegsSoftmax>();
    const int x = warp >> 2, r = tid & (kTile - 1);
    const uint32_t lanes = (uint32_t)(warp & 3) * 32u << 16;
    const uint32_t ts = tmem + x * kTile + lanes, to = tmem + 2 * kTile + x * D + lanes;
    const uint32_t q_at = smem_u32(q_tiles) + (split ? 0u : (uint32_t)x * kTileBytes);
    uint32_t steps_done = 0, count = 0;          // of this tile: scores taken
    for (;; ++taken) {
      if (warp == 0) {                           // (the softmaxes meet at barriers)
        const bool more = take(sh, taken, bad) != nullptr;
        if (lane == 0) sh.softmax_more = more;
      }
      softmax_barrier();
      if (!sh.softmax_more) break;
      const Work p = sh.work[taken % kWorkSlots];
      const int len = p.len, M = p.rows * a.group;
      const int m = p.m0 + (split ? 0 : x * kTile) + r;
      const bool in = m < M;
      const int node = in ? m / a.group : 0;
      const bool live = __any_sync(0xffffffffu, in);
      if (a.parents && p.s1 * kStep > len)
        for (int i = tid; i < p.rows; i += 32 * kSoftmaxWarps)
          sh.parents[i] = a.parents[(size_t)p.b * a.R + i];
      // this thread's row of queries
      float f;
      {
        uint4 w[D / 8];
        const uint4* const src = reinterpret_cast<const uint4*>(
            a.q + (((size_t)p.b * a.R + node) * a.c.kv_heads * a.group +
                   (size_t)p.head * a.group + (in ? m % a.group : 0)) * D);
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          w[i] = in ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
          const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            top = max_nan(top, max_nan(fabsf(bf16_lo(u[k])), fabsf(bf16_hi(u[k]))));
        }
        const QueryScale s(top);
        f = s.factor(a.scale_log2e, exponent_of(a.c, a.layer, 0, p.head));
        const float sign = f < 0.f ? -1.f : 1.f;           // the factor is made positive,
        f = fabsf(f);
        if (f < 1e-37f) f = 1e-37f;                        // and keeps -inf what it is
        if (!(split && x == 1)) {
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const __half2 y = __floats2half2_rn(sign * s.apply(bf16_lo(u[k])),
                                                  sign * s.apply(bf16_hi(u[k])));
              h[k] = *reinterpret_cast<const uint32_t*>(&y);
            }
            sts128(piece_at(q_at, r, i), h[0], h[1], h[2], h[3]);
          }
        }
      }
      async_visible();
      softmax_barrier();                                   // (parents are there, too)
      if (lane == 0) mbar_arrive(&sh.qfull);

      float mref = TV_NEG_INF, l = 0.f;
      int at_node = node;                                  // the path's next node, -1: done
      const int n = p.s1 - p.s0, ops = split ? n : 2 * n;
      for (int i = x; i < ops; i += 2) {
        const int j = split ? i : i >> 1;
        const int pos = (p.s1 - 1 - j) * kStep;
        wait_on(&sh.sfull[x], count & 1, bad);
        tc_fence_after();
        if (live) {
          const uint4 ok = sh.ok[(steps_done + (uint32_t)j) % kOkSlots];
          const bool part = pos + kStep > len || (ok.x & ok.y & ok.z & ok.w) != 0xffffffffu;
          uint32_t see[4] = {ok.x, ok.y, ok.z, ok.w};
          if (pos + kStep > len) {                         // some tokens are the tree's
            uint32_t mine[4];
            const int upto = len - pos + (a.parents ? 0 : node + 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) mine[k] = low_bits(upto, 32 * k);
            if (a.parents) {
              while (at_node >= 0 && len + at_node >= pos) {
                const int bit = len + at_node - pos;
                if (bit < kStep) {
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (bit >> 5 == k) mine[k] |= 1u << (bit & 31);
                }
                const int up = sh.parents[at_node];
                if (in && (at_node == 0 ? up != -1 : up < 0 || up >= at_node))
                  atomicOr(a.status, (uint32_t)TV_STATUS_BAD_TREE);
                at_node = at_node == 0 || up >= at_node ? -1 : max(up, -1);
              }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) see[k] &= mine[k];
          }
          // the largest score
          float top = TV_NEG_INF, top1 = TV_NEG_INF;
          uint32_t c[32];
#pragma unroll 1
          for (int k = 0; k < 4; ++k) {
            tmem_ld32(ts + 32 * k, c);
            const uint32_t now = k == 0 ? see[0] : k == 1 ? see[1] : k == 2 ? see[2] : see[3];
            tmem_wait(c);
            if (part) hide(c, now);
#pragma unroll
            for (int y = 0; y < 32; y += 4) {
              top = fmaxf(fmaxf(top, __uint_as_float(c[y])), __uint_as_float(c[y + 1]));
              top1 = fmaxf(fmaxf(top1, __uint_as_float(c[y + 2])), __uint_as_float(c[y + 3]));
            }
          }
          top = f * fmaxf(top, top1);
          if (__any_sync(0xffffffffu, top > mref + kSlack)) {
            float down = 1.f;
            if (top > mref) {
              down = ex2(mref - top);
              mref = top;
              l *= down;
            }
            if (i >= 2) {                                  // there is a sum to scale
              wait_on(&sh.ofull[x], (count - 1) & 1, bad);
              tc_fence_after();
#pragma unroll 1
              for (int k = 0; k < D / 32; ++k) {
                tmem_ld32(to + 32 * k, c);
                tmem_wait(c);
#pragma unroll
                for (int y = 0; y < 32; ++y) c[y] = __float_as_uint(__uint_as_float(c[y]) * down);
                tmem_st32(to + 32 * k, c);
              }
            }
          }
          const float off = kLift - (mref == TV_NEG_INF ? 0.f : mref);
          const float2 ff = make_float2(f, f), oo = make_float2(off, off);
          float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
          for (int k = 0; k < 4; ++k) {
            tmem_ld32(ts + 32 * k, c);
            const uint32_t now = k == 0 ? see[0] : k == 1 ? see[1] : k == 2 ? see[2] : see[3];
            tmem_wait(c);
            if (part) hide(c, now);
            uint32_t w[16];
#pragma unroll
            for (int y = 0; y < 32; y += 2) {
              float2 e = __ffma2_rn(make_float2(__uint_as_float(c[y]), __uint_as_float(c[y + 1])), ff, oo);
              e.x = ex2(e.x);
              e.y = ex2(e.y);
              acc[(y >> 1) & 1] = __fadd2_rn(acc[(y >> 1) & 1], e);
              const __half2 h = __floats2half2_rn(e.x, e.y);
              w[y >> 1] = *reinterpret_cast<const uint32_t*>(&h);
            }
            tmem_st16(ts + 16 * k, w);
          }
          acc[0] = __fadd2_rn(acc[0], acc[1]);
          l += acc[0].x + acc[0].y;
          tmem_stored();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.pfull[x]);
        ++count;
      }
      steps_done += (uint32_t)n;

      // the sums
      const bool any = x < ops;
      if (any) wait_on(&sh.ofull[x], (count - 1) & 1, bad);
      tc_fence_after();
      float fac[2] = {1.f, 0.f};
      if (split) {
        sh.m[x][r] = any ? mref : TV_NEG_INF;
        sh.l[x][r] = any ? l : 0.f;
        softmax_barrier();
        const float m0 = sh.m[0][r], m1 = sh.m[1][r];
        mref = fmaxf(m0, m1);
        fac[0] = m0 == TV_NEG_INF ? 0.f : ex2(m0 - mref);
        fac[1] = m1 == TV_NEG_INF ? 0.f : ex2(m1 - mref);
        l = sh.l[0][r] * fac[0] + sh.l[1][r] * fac[1];
      }
      const bool whole = p.whole();
      const float inv = !whole ? 1.f
                        : l == 0.f ? 0.f : pow2i(exponent_of(a.c, a.layer, 1, p.head)) / l;
      const size_t slot = 2 * (size_t)blockIdx.x + (p.s0 == 0);
      const int at_row = m - p.m0;
      if (live) {
        // (split: half of the columns each)
        const int c0 = split ? x * (D / 64) : 0, c1 = split ? c0 + D / 64 : D / 32;
        const uint32_t t0 = tmem + 2 * kTile + lanes;
        for (int k = c0; k < c1; ++k) {
          uint32_t c[32];
          float y[32];
          tmem_ld32((split ? t0 : to) + 32 * k, c);
          tmem_wait(c);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            y[i] = split && fac[0] == 0.f ? 0.f : __uint_as_float(c[i]) * fac[0];
          if (split && ops > 1) {
            tmem_ld32(t0 + D + 32 * k, c);
            tmem_wait(c);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              y[i] += fac[1] == 0.f ? 0.f : __uint_as_float(c[i]) * fac[1];
          }
          if (whole) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i] * inv, y[2 * i + 1] * inv);
              w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
            if (in) {
              __nv_bfloat16* const dst =
                  a.out + (((size_t)p.b * a.R + node) * a.c.kv_heads * a.group +
                           (size_t)p.head * a.group + m % a.group) * D + 32 * k;
              if (wide) {
                st_global_32b(dst, w);
                st_global_32b(dst + 16, w + 8);
              } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  reinterpret_cast<uint4*>(dst)[i] =
                      make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
              }
            }
          } else {
            float* const dst = a.part + (slot * 2 * kTile + at_row) * D + 32 * k;
#pragma unroll
            for (int i = 0; i < 32; i += 8)
              st_global_32b(dst + i, reinterpret_cast<const uint32_t*>(y) + i);
          }
        }
        if (!whole && !(split && x == 1)) {
          stats_of(a, D, gridDim.x)[slot * 2 * kTile + at_row] = make_float2(mref, l);
        }
      }
      tc_fence_before();
      give_back(sh, taken);
      softmax_barrier();       // the next piece's queries and sums go where these were
    }
  }
  if (bad) atomicOr(a.status, (uint32_t)TV_STATUS_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc<false>(tmem);
  }
}

// Joins the pieces of an item that spans CTAs: block c * kJoinParts + part takes a part of
// the rows of the item that begins in CTA c and goes on in later ones.
template <int D>
__global__ void __launch_bounds__(256) join_kernel(AttendArgs a, int split, int ctas) {
  asm volatile("griddepcontrol.wait;" ::: "memory");     // (launched before the pieces are there)
  const int c0 = blockIdx.x / kJoinParts, part = blockIdx.x % kJoinParts;
  const Split item = splits_of(a, D, ctas)[c0];
  if (item.b < 0) return;
  const int M = request_of(a, item.b).rows * a.group;
  const float up = pow2i(exponent_of(a.c, a.layer, 1, item.head));
  const int rows = (split ? kTile : 2 * kTile) / kJoinParts;
  const float2* const stats = stats_of(a, D, ctas);
  for (int x = threadIdx.x; x < rows * D / 4; x += blockDim.x) {
    const int row = part * rows + x / (D / 4), col = x % (D / 4) * 4;
    if (item.m0 + row >= M) break;
    float top = TV_NEG_INF, sum = 0.f;
    for (int c = c0; c <= item.last; ++c)
      top = fmaxf(top, stats[((size_t)2 * c + (c == c0)) * 2 * kTile + row].x);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c = c0; c <= item.last; ++c) {
      const size_t at = ((size_t)2 * c + (c == c0)) * 2 * kTile + row;
      const float2 ms = stats[at];
      const float f = ms.y != ms.y ? ms.y : ms.x == TV_NEG_INF ? 0.f : ex2(ms.x - top);
      const float4 v = *reinterpret_cast<const float4*>(a.part + at * D + col);
      sum += f * ms.y;
      y.x += f * v.x;
      y.y += f * v.y;
      y.z += f * v.z;
      y.w += f * v.w;
    }
    store_out(a, item.b, item.head, item.m0 + row, M, col, D, y, sum, up);
  }
}

template <int D>
int launch_tiles(const AttendArgs& a, int sm_count, cudaStream_t stream) {
  const size_t smem = (size_t)(2 + 2 * kStages) * kTile * D * 2 + 1024;
  if (cudaFuncSetAttribute(tile_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           (int)smem) != cudaSuccess) {
    cudaGetLastError();
    return -5;
  }
  const int split = (long long)a.R * a.group <= kTile;
  const int wide = (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
  tile_kernel<D><<<sm_count, kTileThreads, smem, stream>>>(a, split, wide);
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t join = {};
  join.gridDim = dim3((unsigned)(sm_count * kJoinParts));
  join.blockDim = dim3(256);
  join.stream = stream;
  join.attrs = &early;
  join.numAttrs = 1;
  if (cudaGetLastError() != cudaSuccess ||
      cudaLaunchKernelEx(&join, join_kernel<D>, a, split, sm_count) != cudaSuccess) {
    cudaGetLastError();
    return -5;
  }
  return 0;
}

}  // namespace attend
}  // namespace tvk

using namespace tvk::attend;

size_t tv_attend_tile_scratch(int sm_count) {
  return (size_t)sm_count * (2 * 2 * kTile * (128 + 2) * sizeof(float) + sizeof(Split));
}

int tv_launch_attend_tile(const AttendArgs& a, int sm_count, cudaStream_t stream) {
  return a.c.head_dim == 128 ? launch_tiles<128>(a, sm_count, stream)
                             : launch_tiles<64>(a, sm_count, stream);
}
