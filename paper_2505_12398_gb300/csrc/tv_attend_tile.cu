// tv_attend_tile.cu -- attention over the 4-bit key/value cache for many query rows per
// key/value head (sm_103a): large trees and pieces of prompts, on the 5th-generation tensor
// cores.  Mathematics, rounding and the cut into pieces are those of tv_attend.cu.
//
// One persistent CTA per SM, two tiles of 128 rows at a time:
//   warps 0-7, 8-15   softmax of tile 0 and 1, half a row (64 of a step's tokens) per thread:
//                     scores from tensor memory, weights back into it as fp16, over the
//                     first half of the thread's own scores
//   warps 16-19       widen 128 tokens' keys to fp16 in shared memory (a token per thread,
//                     its codes loaded a step ahead), two stages
//   warps 20-23       the same for values
//   warp 24           the products: S = Q K^T (both from shared memory) and O += P V (P
//                     from tensor memory), S and O of both tiles in tensor memory
//   warp 25           the CTA's pieces, in a ring that the others read
//   warps 26, 27      the next piece's queries to fp16 in shared memory as soon as the last
//                     product that reads the present ones is done; at the end, zeros in the
//                     rows behind the requests' last
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
constexpr int kHalfTile = 64;                    // tokens of a thread
constexpr int kSoftmaxWarps = 16;
constexpr int kWidenWarps = 8;                   // four for keys, four for values
constexpr int kMmaWarp = kSoftmaxWarps + kWidenWarps;
constexpr int kQueryWarps = 2;
constexpr int kTileThreads = 32 * (kMmaWarp + 2 + kQueryWarps);
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
constexpr int kTakers = kSoftmaxWarps + kWidenWarps + 1 + kQueryWarps;

struct TileShared {
  uint64_t given[kWorkSlots], taken[kWorkSlots];
  Work work[kWorkSlots];
  int more[2][2];                                // [piece % 2][tile]
  uint64_t kfull[kStages], kempty[kStages], vfull[kStages], vempty[kStages];
  uint64_t sfull[2], pfull[2], ofull[2], qfull, qempty, merge;
  uint32_t tmem;
  // tokens of a step that exist and have a page; a slot is used again four steps later, when
  // both softmaxes are done with it
  alignas(16) uint32_t ok[kOkSlots][4];
  float factor[2][2 * kTile];                    // [piece % 2], of a row's scores
  float top[2][2][kTile], l[2][2][kTile], m[2][kTile];
  Schedule plan;
  int32_t parents[2][1024];                      // [piece % 2]
};

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

// Descriptors of operands whose rows are 128 bytes with the 128-byte swizzle, in two words:
// the start address >> 4 and the leading offset, and what all have (8 rows after 1024 bytes).
// Rows along the other dimension than the sum's (as smem_desc), and rows along the sum's, the
// next 64 columns of the other after kHalfBytes.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t row_desc(const void* p) {
  return (smem_u32(p) >> 4) | (1u << 16);
}
__device__ __forceinline__ uint32_t column_desc(const void* p) {
  return (smem_u32(p) >> 4) | ((kHalfBytes >> 4) << 16);
}
// Instruction descriptor of kind::f16: fp32 accumulator (bits 4-5 = 1), fp16 A and B (0), B by
// columns (bit 16), N >> 3 in bits 17-22, M >> 4 in bits 24-28.
__device__ __forceinline__ constexpr uint32_t f16_desc(int m, int n, bool by_columns) {
  return (1u << 4) | ((by_columns ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(kDescHigh), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 b, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(kDescHigh), "r"(idesc), "r"((uint32_t)accumulate)
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
__device__ __forceinline__ void named_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// Whether any of the 64 threads that share 32 rows says so.
__device__ __forceinline__ bool pair_any(int id, bool say) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)say), "r"(id)
      : "memory");
  return any != 0;
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

// A thread's 64 scores, 16 at a time with the next on their way.  (Not a loop: registers that a
// load is still to fill must not be moved, as they may be from one turn to the next.)
template <typename F>
__device__ __forceinline__ void for_scores(uint32_t ts, F use) {
  uint32_t c[2][16];
  tmem_ld16(ts, c[0]);
#pragma unroll
  for (int k = 0; k < kHalfTile / 16; ++k) {
    uint32_t(&x)[16] = c[k & 1];
    tmem_wait16(x);
    if (k + 1 < kHalfTile / 16) tmem_ld16(ts + 16 * (k + 1), c[(k + 1) & 1]);
    use(k, x);
  }
}
// Scores that a row does not see become -inf in tensor memory; a set bit in `see` is seen.
__device__ __noinline__ void hide_scores(uint32_t ts, uint2 see) {
#pragma unroll 1
  for (int k = 0; k < kHalfTile; k += 16) {
    uint32_t c[16];
    tmem_ld16(ts + k, c);
    tmem_wait16(c);
    const uint32_t bits = (k < 32 ? see.x : see.y) >> (k & 16);
#pragma unroll
    for (int y = 0; y < 16; ++y)
      if (!(bits >> y & 1)) c[y] = 0xff800000u;
    tmem_st16(ts + k, c);
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
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
      mbar_init(&sh.pfull[x], kSoftmaxWarps / 2);
      mbar_init(&sh.ofull[x], 1);
    }
    mbar_init(&sh.qfull, kQueryWarps);
    mbar_init(&sh.qempty, 1 + kSoftmaxWarps);
    mbar_init(&sh.merge, kSoftmaxWarps);
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

  if (warp == kMmaWarp) {
    // ---- products ----
    const uint32_t qd0 = row_desc(q_tiles), qd1 = row_desc(q_tiles + (split ? 0 : kTileBytes));
    const uint32_t kd = row_desc(k_tiles), vd = column_desc(v_tiles);
    uint32_t steps_done = 0, pcount[2] = {0, 0};
    for (; const Work* const w = take(sh, taken, bad); ++taken) {
      const int n = w->s1 - w->s0, ops = split ? n : 2 * n;
      give_back(sh, taken);
      auto step_of = [&](int i) { return steps_done + (uint32_t)(split ? i : i >> 1); };
      auto wait_keys = [&](int i, int x) {
        const uint32_t s = step_of(i);
        if (split || x == 0) wait_on(&sh.kfull[s % kStages], (s / kStages) & 1, bad);
      };
      auto wait_weights = [&](int i, int x) {
        const uint32_t s = step_of(i);
        if (split || x == 0) wait_on(&sh.vfull[s % kStages], (s / kStages) & 1, bad);
        wait_on(&sh.pfull[x], pcount[x] & 1, bad);
        ++pcount[x];
        tc_fence_after();
      };
      auto scores = [&](int i, int x) {
        const uint32_t stage = step_of(i) % kStages;
        if (elect_one()) {
          const uint32_t q = x ? qd1 : qd0, k0 = kd + stage * (kTileBytes >> 4);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = (uint32_t)((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
            mma_ss(tmem + x * kTile, q + off, k0 + off, f16_desc(kTile, kTile, false), k > 0);
          }
          umma_commit<false>(&sh.sfull[x]);
          if (split || x == 1) umma_commit<false>(&sh.kempty[stage]);
          if (i == ops - 1) umma_commit<false>(&sh.qempty);
        }
        __syncwarp();
      };
      auto values = [&](int i, int x) {
        const uint32_t stage = step_of(i) % kStages;
        if (elect_one()) {
          const uint32_t v0 = vd + stage * (kTileBytes >> 4);
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            mma_ts(tmem + 2 * kTile + x * D,
                   tmem + x * kTile + (k >> 2) * kHalfTile + (k & 3) * 8, v0 + k * (2048u >> 4),
                   f16_desc(kTile, D, true), i >= 2 || k > 0);
          umma_commit<false>(&sh.ofull[x]);
          if (split || x == 1) umma_commit<false>(&sh.vempty[stage]);
        }
        __syncwarp();
      };
      // (where the tiles share a step its keys are there long before; where they do not they may
      // come later than the weights)
      auto turn = [&](int i, int x) {
        const bool next = i + 2 < ops;
        if (next && !split) wait_keys(i + 2, x);
        wait_weights(i, x);
        values(i, x);
        if (next) {
          if (split) {
            wait_keys(i + 2, x);
            tc_fence_after();
          }
          scores(i + 2, x);
        }
      };
      wait_on(&sh.qfull, taken & 1, bad);
      wait_keys(0, 0);
      tc_fence_after();
      scores(0, 0);
      if (ops > 1) {
        wait_keys(1, 1);
        tc_fence_after();
        scores(1, 1);
      }
      for (int i = 0; i < ops; i += 2) {
        turn(i, 0);
        if (i + 1 < ops) turn(i + 1, 1);
      }
      steps_done += (uint32_t)n;
    }
  } else if (warp == kMmaWarp + 1) {
    // ---- pieces ----
    if (lane == 0) {
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
    }
  } else if (warp > kMmaWarp + 1) {
    // ---- queries: a row by D / 8 lanes, 8 columns each ----
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kAhead = 4;
    const int me = warp - (kMmaWarp + 2), col = lane % kLanes;
    for (; const Work* const w = take(sh, taken, bad); ++taken) {
      const Work p = *w;
      give_back(sh, taken);
      const int M = p.rows * a.group;
      const int key_exponent = exponent_of(a.c, a.layer, 0, p.head);
      wait_on(&sh.qempty, (taken & 1) ^ 1, bad);
      if (a.parents && p.s1 * kStep > p.len)
        for (int i = lane + 32 * me; i < p.rows; i += 32 * kQueryWarps)
          sh.parents[taken & 1][i] = a.parents[(size_t)p.b * a.R + i];
      // (rows behind the last stay as they are: nothing of theirs is stored)
      const int rows = min(rows_of_item, M - p.m0);
      for (int r0 = me * kRows; r0 < rows; r0 += kQueryWarps * kRows * kAhead) {
        uint4 w4[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int r = min(r0 + k * kQueryWarps * kRows + lane / kLanes, rows - 1), m = p.m0 + r;
          w4[k] = __ldg(reinterpret_cast<const uint4*>(
                            a.q + (((size_t)p.b * a.R + m / a.group) * a.c.kv_heads * a.group +
                                   (size_t)p.head * a.group + m % a.group) * D) + col);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int r = min(r0 + k * kQueryWarps * kRows + lane / kLanes, rows - 1);
          const uint32_t u[4] = {w4[k].x, w4[k].y, w4[k].z, w4[k].w};
          float top = 0.f;
#pragma unroll
          for (int y = 0; y < 4; ++y)
            top = max_nan(top, max_nan(fabsf(bf16_lo(u[y])), fabsf(bf16_hi(u[y]))));
#pragma unroll
          for (int d = kLanes / 2; d > 0; d >>= 1)
            top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
          const QueryScale s(top);
          float f = s.factor(a.scale_log2e, key_exponent);
          const float sign = f < 0.f ? -1.f : 1.f;         // the factor is made positive,
          f = fabsf(f);
          if (f < 1e-37f) f = 1e-37f;                      // and keeps -inf what it is
          uint32_t h[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const __half2 z = __floats2half2_rn(sign * s.apply(bf16_lo(u[y])),
                                                sign * s.apply(bf16_hi(u[y])));
            h[y] = *reinterpret_cast<const uint32_t*>(&z);
          }
          sts128(piece_at(smem_u32(q_tiles) + (uint32_t)(r >> 7) * kTileBytes, r & (kTile - 1),
                          col),
                 h[0], h[1], h[2], h[3]);
          if (col == 0) sh.factor[taken & 1][r] = f;
        }
      }
      async_visible();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.qfull);
    }
    zero_rows(a, D, (int)blockIdx.x * kQueryWarps + me, (int)gridDim.x * kQueryWarps);
  } else if (warp >= kSoftmaxWarps) {
    // ---- keys and values to fp16 ----
    const int side = warp >= kSoftmaxWarps + 4, row = tid & (kTile - 1);
    uint64_t* const full = side ? sh.vfull : sh.kfull;
    uint64_t* const empty = side ? sh.vempty : sh.kempty;
    const uint32_t base = smem_u32(side ? v_tiles : k_tiles);
    uint32_t s = 0;
    for (; const Work* const w = take(sh, taken, bad); ++taken) {
      const Work p = *w;
      give_back(sh, taken);
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
          if (lane == 0) sh.ok[s % kOkSlots][warp & 3] = word;
          if (!now.there && step * kStep + row < p.tokens)
            atomicOr(a.status, (uint32_t)TV_STATUS_BAD_PAGE);
        }
        async_visible();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[stage]);
      }
    }
  } else {
    // ---- softmax ----
    const int x = warp >> 3, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane;
    const int tile_id = 1 + x, pair_id = 4 + 4 * x + (warp & 3);         // barriers
    const uint32_t lanes = (uint32_t)(warp & 3) * 32u << 16;
    const uint32_t ts = tmem + x * kTile + half * kHalfTile + lanes;
    const uint32_t to = tmem + 2 * kTile + x * D + half * (D / 2) + lanes;
    uint32_t steps_done = 0, count = 0, merged = 0;        // count: scores of this tile taken
    for (;; ++taken) {
      if ((warp & 7) == 0) {                     // (a tile's warps meet at barriers)
        const bool more = take(sh, taken, bad) != nullptr;
        if (lane == 0) sh.more[taken & 1][x] = more;
      }
      named_barrier(tile_id, 16 * kSoftmaxWarps);
      if (!sh.more[taken & 1][x]) break;
      const Work p = sh.work[taken % kWorkSlots];
      give_back(sh, taken);
      const int len = p.len, M = p.rows * a.group;
      const int m = p.m0 + (split ? 0 : x * kTile) + r;
      const bool in = m < M;
      const int node = in ? m / a.group : 0;
      const bool live = __any_sync(0xffffffffu, in);
      const int32_t* const parents = sh.parents[taken & 1];
      wait_on(&sh.qfull, taken & 1, bad);
      const float f = in ? sh.factor[taken & 1][(split ? 0 : x * kTile) + r] : 1e-37f;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.qempty);

      float mref = TV_NEG_INF, l = 0.f;
      int at_node = node;                                  // the path's next node, -1: done
      const int n = p.s1 - p.s0, ops = split ? n : 2 * n;
      for (int i = x; i < ops; i += 2) {
        const int j = split ? i : i >> 1;
        const int pos = (p.s1 - 1 - j) * kStep;
        wait_on(&sh.sfull[x], count & 1, bad);
        tc_fence_after();
        if (live) {
          uint2 see = *reinterpret_cast<const uint2*>(
              &sh.ok[(steps_done + (uint32_t)j) % kOkSlots][2 * half]);
          if (pos + kStep > len) {                         // some tokens are the tree's
            const int from = pos + half * kHalfTile;
            const int upto = len - from + (a.parents ? 0 : node + 1);
            uint2 mine = make_uint2(low_bits(upto, 0), low_bits(upto, 32));
            if (a.parents) {
              while (at_node >= 0 && len + at_node >= pos) {
                const int bit = len + at_node - from;
                if (bit >= 0 && bit < 32) mine.x |= 1u << bit;
                if (bit >= 32 && bit < 64) mine.y |= 1u << (bit - 32);
                const int up = parents[at_node];
                if (in && (at_node == 0 ? up != -1 : up < 0 || up >= at_node))
                  atomicOr(a.status, (uint32_t)TV_STATUS_BAD_TREE);
                at_node = at_node == 0 || up >= at_node ? -1 : max(up, -1);
              }
            }
            see.x &= mine.x;
            see.y &= mine.y;
          }
          if (__any_sync(0xffffffffu, (see.x & see.y) != 0xffffffffu)) hide_scores(ts, see);
          // the largest score of this half
          float top2[2] = {TV_NEG_INF, TV_NEG_INF};
          for_scores(ts, [&](int, const uint32_t (&c)[16]) {
#pragma unroll
            for (int y = 0; y < 16; y += 4) {
              top2[0] = fmaxf(fmaxf(top2[0], __uint_as_float(c[y])), __uint_as_float(c[y + 1]));
              top2[1] = fmaxf(fmaxf(top2[1], __uint_as_float(c[y + 2])),
                              __uint_as_float(c[y + 3]));
            }
          });
          // (lanes without a row hold scores of whatever was there, and have no say)
          float top = in ? f * fmaxf(top2[0], top2[1]) : TV_NEG_INF;
          // weights are relative to what the largest score was, until it has grown too far
          if (pair_any(pair_id, top > mref + kSlack)) {
            sh.top[x][half][r] = top;
            named_barrier(pair_id, 64);
            top = fmaxf(top, sh.top[x][half ^ 1][r]);
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
              for (int k = 0; k < D / 2; k += 32) {
                uint32_t c[32];
                tmem_ld32(to + k, c);
                tmem_wait(c);
#pragma unroll
                for (int y = 0; y < 32; ++y) c[y] = __float_as_uint(__uint_as_float(c[y]) * down);
                tmem_st32(to + k, c);
              }
            }
          }
          const float off = kLift - (mref == TV_NEG_INF ? 0.f : mref);
          const float2 ff = make_float2(f, f), oo = make_float2(off, off);
          float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          uint32_t w[16];
          for_scores(ts, [&](int k, const uint32_t (&c)[16]) {
#pragma unroll
            for (int y = 0; y < 16; y += 2) {
              float2 e = __ffma2_rn(
                  make_float2(__uint_as_float(c[y]), __uint_as_float(c[y + 1])), ff, oo);
              e.x = ex2(e.x);
              e.y = ex2(e.y);
              acc[(y >> 1) & 1] = __fadd2_rn(acc[(y >> 1) & 1], e);
              const __half2 h = __floats2half2_rn(e.x, e.y);
              w[8 * (k & 1) + (y >> 1)] = *reinterpret_cast<const uint32_t*>(&h);
            }
            if (k & 1) tmem_st16(ts + 8 * (k - 1), w);
          });
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
      if (x < ops) wait_on(&sh.ofull[x], (count - 1) & 1, bad);
      tc_fence_after();
      sh.l[x][half][r] = x < ops ? l : 0.f;
      float fac[2] = {1.f, 0.f};
      if (split) {
        if (half == 0) sh.m[x][r] = x < ops ? mref : TV_NEG_INF;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.merge);
        wait_on(&sh.merge, merged++ & 1, bad);
        const float m0 = sh.m[0][r], m1 = sh.m[1][r];
        mref = fmaxf(m0, m1);
        fac[0] = m0 == TV_NEG_INF ? 0.f : ex2(m0 - mref);
        fac[1] = m1 == TV_NEG_INF ? 0.f : ex2(m1 - mref);
        l = (sh.l[0][0][r] + sh.l[0][1][r]) * fac[0] + (sh.l[1][0][r] + sh.l[1][1][r]) * fac[1];
      } else {
        named_barrier(pair_id, 64);
        l = sh.l[x][0][r] + sh.l[x][1][r];
      }
      if (live && !(split && x == 1)) {          // (tile 0's threads read both tiles' sums)
        const bool whole = p.whole();
        const float inv = !whole ? 1.f
                          : l == 0.f ? 0.f
                                     : pow2i(exponent_of(a.c, a.layer, 1, p.head)) / l;
        const size_t row = (2 * (size_t)blockIdx.x + (p.s0 == 0)) * 2 * kTile + (m - p.m0);
        fac[0] *= inv;
        fac[1] *= inv;
#pragma unroll 1
        for (int k = 0; k < D / 2; k += 32) {
          const int col = half * (D / 2) + k;
          uint32_t c[32];
          tmem_ld32(to + k, c);
          tmem_wait(c);
#pragma unroll
          for (int y = 0; y < 32; ++y)
            c[y] = split && fac[0] == 0.f ? 0u : __float_as_uint(__uint_as_float(c[y]) * fac[0]);
          if (split && ops > 1) {
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              uint32_t d[16];
              tmem_ld16(to + D + k + 16 * z, d);
              tmem_wait16(d);
#pragma unroll
              for (int y = 0; y < 16; ++y)
                c[16 * z + y] = __float_as_uint(
                    __uint_as_float(c[16 * z + y]) +
                    (fac[1] == 0.f ? 0.f : __uint_as_float(d[y]) * fac[1]));
            }
          }
          if (whole) {
            uint32_t w[16];
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(c[2 * y]),
                                                             __uint_as_float(c[2 * y + 1]));
              w[y] = *reinterpret_cast<const uint32_t*>(&h);
            }
            if (in) {
              __nv_bfloat16* const dst =
                  a.out + (((size_t)p.b * a.R + node) * a.c.kv_heads * a.group +
                           (size_t)p.head * a.group + m % a.group) * D + col;
              if (wide) {
                st_global_32b(dst, w);
                st_global_32b(dst + 16, w + 8);
              } else {
#pragma unroll
                for (int y = 0; y < 4; ++y)
                  reinterpret_cast<uint4*>(dst)[y] =
                      make_uint4(w[4 * y], w[4 * y + 1], w[4 * y + 2], w[4 * y + 3]);
              }
            }
          } else if (in) {
#pragma unroll
            for (int y = 0; y < 32; y += 8) st_global_32b(a.part + row * D + col + y, c + y);
          }
        }
        if (!whole && half == 0 && in) stats_of(a, D, gridDim.x)[row] = make_float2(mref, l);
      }
      tc_fence_before();
      if (split) {                               // both tiles' sums may be overwritten
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.merge);
        wait_on(&sh.merge, merged++ & 1, bad);
      }
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
