// tv_attend_tile.cu -- attention over the 4-bit key/value cache for many query rows per
// key/value head (sm_103a): large trees and pieces of prompts, on the 5th-generation tensor
// cores.  Mathematics, rounding and the cut into pieces are those of tv_attend.cu.
//
// One persistent CTA per SM, two tiles of 128 rows at a time:
//   warps 0-3, 4-7    softmax of tile 0 and 1, one row per thread: a step's 128 scores from
//                     tensor memory, 32 at a time with the next on their way, and weights back
//                     into it as fp16, those of 64 tokens over the first half of their scores
//   warps 8-11        widen 128 tokens' keys to fp16 in shared memory (a token per thread,
//                     its codes loaded a step ahead), two stages
//   warps 12-15       the same for values
//   warps 16, 17      the products of tile 0 and 1: S = Q K^T (both from shared memory) and
//                     O += P V (P from tensor memory), S and O in tensor memory
//   warp 18           the CTA's pieces, in a ring that the others read
//   warp 19           zeros in the rows behind the requests' last
// (registers that the others leave go to the softmax).  The softmax threads also bring their rows
// of queries to shared memory: two warps beside them took 24 thousand clocks for 256 rows.
// The two tiles take turns: while one's scores become weights, the tensor cores work on the
// other.  (A warp's products are issued little faster than they run, and each barrier that it
// tests takes 100 clocks: with one warp for both tiles the tensor cores had half of the time
// nothing to do.)  Where an item has 128 rows or fewer both tiles are the same rows and take
// alternate steps, and their sums are joined at the end.
// Steps go from the last tokens to the first, so that a row's path to the root is walked once,
// and the tree's tokens, which rows see in part, come first.
//
// A product that overwrites a tile's scores waits until the one that reads its weights has ended
// (1 % of the time).  Where a product's operands were not known to be the warp's, its issue took
// as long as the product: 432 us for 406 at 128 trees of 61 rows over 4096 tokens.  Scores by 64
// tokens, made while the softmax works on the other 64, took as long (404 us there, but
// 178 for 172 of prompts): with 64 columns a product is bound by shared memory.  Every wait is
// bounded; one that gives up raises the timeout status, and the loops go on to their end.
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
constexpr int kHalfTile = 64;                    // tokens whose weights are handed over at once
constexpr int kSoftmaxWarps = 8;
constexpr int kWidenWarps = 8;                   // four for keys, four for values
constexpr int kMmaWarp = kSoftmaxWarps + kWidenWarps;
constexpr int kPieceWarp = kMmaWarp + 2;
constexpr int kTileThreads = 32 * (kPieceWarp + 2);
// registers per thread after the split
constexpr int kRegsSoftmax = 144, kRegsWiden = 64, kRegsOther = 64, kRegsLaunch = 96;
static_assert(32 * (kSoftmaxWarps * kRegsSoftmax + kWidenWarps * kRegsWiden + 4 * kRegsOther) <=
                  kTileThreads * kRegsLaunch,
              "the warpgroups' registers fit what the block was launched with");
constexpr int kStages = 2;
constexpr int kOkSlots = 4;
constexpr uint32_t kHalfBytes = kTile * 128;     // 64 columns (128 bytes) of a tile's rows

// An item that begins in a CTA and goes on in later ones, up to `last`; b < 0: there is none.
struct Split {
  int b, head, m0, last;
};

// A piece as the warps take it; more = 0: there is none.
struct Work {
  int more, b, head, m0, s0, s1, steps, tokens, len, rows;
  __device__ __forceinline__ bool whole() const { return s0 == 0 && s1 == steps; }
};
constexpr int kPieceSlots = 4;
constexpr int kTakers = 2 + kWidenWarps + 2;       // (of the softmax one of each tile)

struct TileShared {
  uint64_t given[kPieceSlots], taken[kPieceSlots];
  Work work[kPieceSlots];
  Work now[2][2];                                // [tile][piece % 2], the softmax's
  uint64_t kfull[kStages], kempty[kStages], vfull[kStages], vempty[kStages];
  uint64_t sfull[2], pfull[2][2], ofull[2][2];   // [tile][half of the tokens]
  uint64_t qfull[2], merge;
  uint32_t tmem;
  // tokens of a step that exist and have a page; a slot is used again four steps later, when
  // both softmaxes are done with it
  alignas(16) uint32_t ok[kOkSlots][4];
  float m[2][kTile], l[2][kTile];
  Schedule plan;
  int32_t parents[2][1024];                      // [tile]
};

template <int kRegs>
__device__ __forceinline__ void regs_fewer() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void regs_more() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}

// The n-th piece.  Whether there is one is only one thread's or one warp's to say: after a
// wait that gave up others may see something else.
__device__ __forceinline__ const Work* take(TileShared& sh, uint32_t n, uint32_t& bad) {
  wait_on(&sh.given[n % kPieceSlots], (n / kPieceSlots) & 1, bad);
  const Work* const w = &sh.work[n % kPieceSlots];
  return __all_sync(0xffffffffu, !bad && w->more) ? w : nullptr;
}
__device__ __forceinline__ void give_back(TileShared& sh, uint32_t n) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.taken[n % kPieceSlots]);
}

// What all lanes of a warp hold alike, known as such to the compiler: a product takes its operands
// from registers of the whole warp.
template <typename T>
__device__ __forceinline__ T uniform(T x) {
  return __shfl_sync(0xffffffffu, x, 0);
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
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c,
                                       uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c),
               "r"(d)
               : "memory");
}
__device__ __forceinline__ uint4 lds128_at(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(at)
               : "memory");
  return v;
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
  __device__ __forceinline__ void load(const AttendArgs& a, const Work& p, int page, int pos,
                                       int side) {
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

// The lowest n of 64 bits.
__device__ __forceinline__ unsigned long long low_bits64(int n) {
  return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1ull;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Scales a row's sums.
template <int D>
__device__ __noinline__ void scale_sums(uint32_t to, float down) {
#pragma unroll 1
  for (int k = 0; k < D; k += 16) {
    uint32_t d[16];
    tmem_ld16(to + k, d);
    tmem_wait16(d);
#pragma unroll
    for (int y = 0; y < 16; ++y) d[y] = __float_as_uint(__uint_as_float(d[y]) * down);
    tmem_st16(to + k, d);
  }
  tmem_stored();
}
// Scores that a row does not see become -inf in tensor memory; a set bit in `see` is seen.
// (Apart, and there: in the registers of the weights' loop it takes that loop's.)
__device__ __noinline__ void hide_scores(uint32_t ts, uint4 see) {
#pragma unroll 1
  for (int k = 0; k < kTile; k += 32) {
    uint32_t c[32];
    tmem_ld32(ts + k, c);
    tmem_wait(c);
    const uint32_t on = k < 64 ? (k < 32 ? see.x : see.y) : (k < 96 ? see.z : see.w);
#pragma unroll
    for (int y = 0; y < 32; ++y)
      if (!(on >> y & 1)) c[y] = 0xff800000u;
    tmem_st32(ts + k, c);
  }
  tmem_stored();
}

// The scratch: two pieces of every CTA, their rows' (maximum, sum), the CTAs' split items.
__device__ __forceinline__ float2* stats_of(const AttendArgs& a, int D, int ctas) {
  return reinterpret_cast<float2*>(a.part + (size_t)2 * ctas * 2 * kTile * D);
}
__device__ __forceinline__ Split* splits_of(const AttendArgs& a, int D, int ctas) {
  return reinterpret_cast<Split*>(stats_of(a, D, ctas) + (size_t)2 * ctas * 2 * kTile);
}

template <int D>
__global__ void __launch_bounds__(kTileThreads, 1) tile_kernel(AttendArgs a, int split) {
  constexpr uint32_t kTileBytes = kTile * D * 2;
  extern __shared__ uint8_t smem_raw[];
  __shared__ TileShared sh;
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* const q_tiles = smem;                               // [2]
  uint8_t* const k_tiles = smem + 2 * kTileBytes;              // [kStages]
  uint8_t* const v_tiles = k_tiles + kStages * kTileBytes;
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
  const int rows_of_item = split ? kTile : 2 * kTile;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.kfull[i], 4);
      mbar_init(&sh.kempty[i], split ? 1 : 2);
      mbar_init(&sh.vfull[i], 4);
      mbar_init(&sh.vempty[i], split ? 1 : 2);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sh.sfull[x], 1);
      for (int i = 0; i < 2; ++i) mbar_init(&sh.pfull[x][i], kSoftmaxWarps / 2);
      for (int i = 0; i < 2; ++i) mbar_init(&sh.ofull[x][i], 1);
      mbar_init(&sh.qfull[x], split ? kSoftmaxWarps : kSoftmaxWarps / 2);
    }
    mbar_init(&sh.merge, kSoftmaxWarps);
    for (int i = 0; i < kPieceSlots; ++i) {
      mbar_init(&sh.given[i], 1);
      mbar_init(&sh.taken[i], kTakers);
    }
    fence_mbar_init();
  }
  if (warp == kMmaWarp) tmem_alloc<false>(&sh.tmem);
  Walker walker;
  // (61 rows of 8000 tokens and one head: 48.5 us with one step at least, 34.4 with two; of 2000
  // and 8 heads 29.5 and 34.8)
  const Shares shares = plan(a, sh.plan, rows_of_item, blockIdx.x, gridDim.x, 12.f, walker);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(sh.tmem);
  uint32_t bad = 0, taken = 0;                   // pieces so far

  if (warp >= kMmaWarp) regs_fewer<kRegsOther>();
  if (warp >= kMmaWarp && warp < kPieceWarp) {
    // ---- products ----
    const int x = warp - kMmaWarp;
    const uint32_t qd = row_desc(q_tiles + (split ? 0 : x * kTileBytes));
    const uint32_t kd = row_desc(k_tiles), vd = column_desc(v_tiles);
    const uint32_t ts = tmem + x * kTile, to = tmem + 2 * kTile + x * D;
    uint32_t steps_done = 0, count = 0;          // count: weights of this tile taken
    for (; const Work* const w = take(sh, taken, bad); ++taken) {
      const int n = uniform(w->s1 - w->s0), stride = split ? 2 : 1, first = split ? x : 0;
      give_back(sh, taken);
      auto scores = [&](int j) {
        const uint32_t s = steps_done + (uint32_t)j, stage = s % kStages;
        wait_on(&sh.kfull[stage], (s / kStages) & 1, bad);
        tc_fence_after();
        if (elect_one()) {
          const uint32_t k0 = kd + stage * (kTileBytes >> 4);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = (uint32_t)((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
            mma_ss(ts, qd + off, k0 + off, f16_desc(kTile, kTile, false), k > 0);
          }
          umma_commit<false>(&sh.sfull[x]);
          umma_commit<false>(&sh.kempty[stage]);
        }
        __syncwarp();
      };
      wait_on(&sh.qfull[split ? 0 : x], taken & 1, bad);
      if (first < n) scores(first);
      for (int j = first; j < n; j += stride, ++count) {
        const uint32_t s = steps_done + (uint32_t)j, stage = s % kStages;
        wait_on(&sh.vfull[stage], (s / kStages) & 1, bad);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          wait_on(&sh.pfull[x][half], count & 1, bad);
          tc_fence_after();
          if (elect_one()) {
            const uint32_t v0 =
                vd + stage * (kTileBytes >> 4) + half * ((kHalfTile * 128u) >> 4);
#pragma unroll
            for (int k = 0; k < kHalfTile / 16; ++k)
              mma_ts(to, ts + half * kHalfTile + k * 8, v0 + k * (2048u >> 4),
                     f16_desc(kTile, D, true), j > first || half > 0 || k > 0);
            umma_commit<false>(&sh.ofull[x][half]);
            if (half) umma_commit<false>(&sh.vempty[stage]);
          }
          __syncwarp();
        }
        wait_on(&sh.ofull[x][1], count & 1, bad);
        if (j + stride < n) scores(j + stride);
      }
      steps_done += (uint32_t)n;
    }
  } else if (warp == kPieceWarp) {
    // ---- pieces ----
    if (lane == 0) {
      Piece p;
      Split split_item = {-1, 0, 0, 0};
      for (uint32_t n = 0;; ++n) {
        wait_on(&sh.taken[n % kPieceSlots], ((n / kPieceSlots) & 1) ^ 1, bad);
        Work w = {};
        if (!bad && walker.next(a, rows_of_item, p)) {
          w = Work{1, p.b, p.head, p.m0, p.s0, p.s1, p.steps, p.tokens, p.rq.len, p.rq.rows};
          if (p.s0 == 0 && p.s1 < p.steps)
            split_item = Split{p.b, p.head, p.m0, shares.owner(p.first + p.steps - 1)};
        }
        sh.work[n % kPieceSlots] = w;
        mbar_arrive(&sh.given[n % kPieceSlots]);
        if (!w.more) break;
      }
      splits_of(a, D, gridDim.x)[blockIdx.x] = split_item;
    }
  } else if (warp > kPieceWarp) {
    zero_rows(a, D, (int)blockIdx.x, (int)gridDim.x);
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
      give_back(sh, taken);
      auto page_at = [&](int step) {
        const int pos = step * kStep + row;
        return step >= p.s0 && pos < p.tokens ? page_of(a.c, a.t, p.b, pos) : -1;
      };
      int page_next = page_at(p.s1 - 2);
      Token<D> token;
      token.load(a, p, page_at(p.s1 - 1), (p.s1 - 1) * kStep + row, side);
      for (int step = p.s1 - 1; step >= p.s0; --step, ++s) {
        const uint32_t stage = s % kStages;
        wait_on(&empty[stage], ((s / kStages) & 1) ^ 1, bad);
        token.widen_to(base + stage * kTileBytes, row);
        if (!side) {
          const uint32_t word = __ballot_sync(0xffffffffu, token.there);
          if (lane == 0) sh.ok[s % kOkSlots][warp & 3] = word;
          if (!token.there && step * kStep + row < p.tokens)
            atomicOr(a.status, (uint32_t)TV_STATUS_BAD_PAGE);
        }
        async_visible();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[stage]);
        token.load(a, p, page_next, (step - 1) * kStep + row, side);
        page_next = page_at(step - 2);
      }
    }
  } else {
    // ---- softmax ----
    regs_more<kRegsSoftmax>();
    const int x = warp >> 2, r = tid & (kTile - 1);
    const uint32_t lanes = (uint32_t)(warp & 3) * 32u << 16;
    const uint32_t ts = tmem + x * kTile + lanes, to = tmem + 2 * kTile + x * D + lanes;
    uint32_t steps_done = 0, count = 0, merged = 0;        // count: scores of this tile taken
    // the next piece; false: there is none.  (A tile's warps meet at barriers, so one of them
    // says it for all.)
    auto take_next = [&]() -> bool {
      Work& w = sh.now[x][taken & 1];
      if ((warp & 3) == 0) {
        const bool more = take(sh, taken, bad) != nullptr;
        if (lane == 0) {
          w = sh.work[taken % kPieceSlots];
          w.more = more;
        }
        give_back(sh, taken);
      }
      named_barrier(1 + x, 16 * kSoftmaxWarps);
      ++taken;
      return w.more;
    };
    // A warp's 32 rows of queries come, and its rows of sums go, through its rows of a tile of
    // queries, so that lanes beside one another have pieces of one row: a row for each lane
    // takes L1 32 lines at once (5 and 4 thousand clocks a piece, 2 and 2 so).
    const uint32_t mine = smem_u32(q_tiles) + (uint32_t)x * kTileBytes;
    const int w0 = (warp & 3) * 32;
    // rows of all heads before this thread's one of a request
    auto row_of = [&](const Work& w) {
      const int m = min(w.m0 + (split ? 0 : x * kTile) + r, w.rows * a.group - 1);
      const int i = m / a.group;
      return (i * a.c.kv_heads + w.head) * a.group + (m - i * a.group);
    };
    bool more = take_next();
    while (more) {
      const Work& p = sh.now[x][(taken - 1) & 1];
      const int len = p.len, M = p.rows * a.group, top_step = p.s1 - 1;
      const int m = p.m0 + (split ? 0 : x * kTile) + r;
      const bool in = m < M;
      const int node = in ? m / a.group : 0;
      const bool live = __any_sync(0xffffffffu, in);
      const int row = row_of(p);
      const int32_t* const parents = sh.parents[x];
      if (a.parents && p.s1 * kStep > len)
        for (int i = r; i < p.rows; i += kTile)
          sh.parents[x][i] = a.parents[(size_t)p.b * a.R + i];
      float f;
      {
        constexpr int kLanes = D / 8, kRows = 32 / kLanes;
        const uint4* const src = reinterpret_cast<const uint4*>(a.q) +
                                 (size_t)p.b * a.R * a.c.kv_heads * a.group * kLanes +
                                 lane % kLanes;
        uint4 q[D / 8];
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {        // (32 / kRows = D / 8 loads)
          const int from = __shfl_sync(0xffffffffu, row, k * kRows + lane / kLanes);
          q[k] = __ldg(src + (size_t)from * kLanes);
        }
#pragma unroll
        for (int k = 0; k < D / 8; ++k)
          sts128(piece_at(mine, w0 + k * kRows + lane / kLanes, lane % kLanes), q[k].x, q[k].y,
                 q[k].z, q[k].w);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < D / 8; ++k) q[k] = lds128_at(piece_at(mine, r, k));
        uint32_t top2 = 0;                       // largest magnitudes of two columns, in bf16
#pragma unroll
        for (int k = 0; k < D / 8; ++k)
          top2 = max_nan_bf16x2(max_nan_bf16x2(top2, q[k].x & 0x7fff7fffu),
                                max_nan_bf16x2(q[k].y & 0x7fff7fffu,
                                               max_nan_bf16x2(q[k].z & 0x7fff7fffu,
                                                              q[k].w & 0x7fff7fffu)));
        const QueryScale s(max_nan(bf16_lo(top2), bf16_hi(top2)));
        f = s.factor(a.scale_log2e, exponent_of(a.c, a.layer, 0, p.head));
        const float up0 = f < 0.f ? -s.up0 : s.up0;        // the factor is made positive,
        f = fabsf(f);
        if (f < 1e-37f || !in) f = 1e-37f;                 // and keeps -inf what it is
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          if (split && x == 1) break;            // (both tiles take the first's)
          const uint32_t u[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
          uint32_t h[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const __half2 z = __floats2half2_rn(bf16_lo(u[y]) * up0 * s.up1,
                                                bf16_hi(u[y]) * up0 * s.up1);
            h[y] = *reinterpret_cast<const uint32_t*>(&z);
          }
          sts128(piece_at(mine, r, k), h[0], h[1], h[2], h[3]);
        }
      }
      async_visible();
      named_barrier(1 + x, 16 * kSoftmaxWarps);            // (the parents are there, too)
      if (lane == 0) mbar_arrive(&sh.qfull[split ? 0 : x]);

      float mref = TV_NEG_INF, l = 0.f;
      int at_node = node;                                  // the path's next node, -1: done
      const int n = p.s1 - p.s0, ops = split ? n : 2 * n;
      for (int i = x; i < ops; i += 2, ++count) {
        const int j = split ? i : i >> 1;
        const int pos = (top_step - j) * kStep;
        wait_on(&sh.sfull[x], count & 1, bad);
        tc_fence_after();
        if (live) {
          uint4 see = *reinterpret_cast<const uint4*>(
              sh.ok[(steps_done + (uint32_t)j) % kOkSlots]);
          if (pos + kStep > len) {                         // some tokens are the tree's
            const int upto = len - pos + (a.parents ? 0 : node + 1);
            unsigned long long lower = low_bits64(upto), upper = low_bits64(upto - 64);
            if (a.parents) {
              while (at_node >= 0 && len + at_node >= pos) {
                const int bit = len + at_node - pos;
                const unsigned long long on = 1ull << (bit & 63);
                if (bit < 64)
                  lower |= on;
                else if (bit < 128)
                  upper |= on;
                const int up = parents[at_node];
                if (in && (at_node == 0 ? up != -1 : up < 0 || up >= at_node))
                  atomicOr(a.status, (uint32_t)TV_STATUS_BAD_TREE);
                at_node = at_node == 0 || up >= at_node ? -1 : max(up, -1);
              }
            }
            see.x &= (uint32_t)lower;
            see.y &= (uint32_t)(lower >> 32);
            see.z &= (uint32_t)upper;
            see.w &= (uint32_t)(upper >> 32);
          }
          if (__any_sync(0xffffffffu, (see.x & see.y & see.z & see.w) != 0xffffffffu))
            hide_scores(ts, see);
          const float2 ff = make_float2(f, f);
          float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          uint32_t c[2][32], w[32];
          tmem_ld32(ts, c[0]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t(&z)[32] = c[k & 1];
            tmem_wait(z);
            if (k < 3) tmem_ld32(ts + 32 * (k + 1), c[(k + 1) & 1]);
            float top2[2] = {TV_NEG_INF, TV_NEG_INF};
#pragma unroll
            for (int y = 0; y < 32; y += 4) {
              top2[0] = fmaxf(fmaxf(top2[0], __uint_as_float(z[y])), __uint_as_float(z[y + 1]));
              top2[1] = fmaxf(fmaxf(top2[1], __uint_as_float(z[y + 2])),
                              __uint_as_float(z[y + 3]));
            }
            // (lanes without a row hold scores of whatever was there, and have no say)
            const float top = in ? f * fmaxf(top2[0], top2[1]) : TV_NEG_INF;
            // weights are relative to what the largest score was, until it has grown too far
            if (__any_sync(0xffffffffu, top > mref + kSlack)) {
              // (the next scores are on their way to registers that a call may move)
              if (k < 3) tmem_wait(c[(k + 1) & 1]);
              float down = 1.f;
              if (top > mref) {
                down = ex2(mref - top);
                mref = top;
              }
              l *= down;
              acc[0] = make_float2(acc[0].x * down, acc[0].y * down);
              acc[1] = make_float2(acc[1].x * down, acc[1].y * down);
              if (k & 1) {                       // weights that were not handed over yet
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                  const float2 e = widen(w[y]);
                  const __half2 h = __floats2half2_rn(e.x * down, e.y * down);
                  w[y] = *reinterpret_cast<const uint32_t*>(&h);
                }
              }
              if (i >= 2 || k >= 2) {            // there is a sum to scale
                if (k < 2)
                  wait_on(&sh.ofull[x][1], (count - 1) & 1, bad);
                else
                  wait_on(&sh.ofull[x][0], count & 1, bad);
                tc_fence_after();
                scale_sums<D>(to, down);
              }
            }
            const float off = kLift - (mref == TV_NEG_INF ? 0.f : mref);
            const float2 oo = make_float2(off, off);
#pragma unroll
            for (int y = 0; y < 32; y += 2) {
              float2 e = __ffma2_rn(
                  make_float2(__uint_as_float(z[y]), __uint_as_float(z[y + 1])), ff, oo);
              e.x = ex2(e.x);
              e.y = ex2(e.y);
              acc[(y >> 1) & 1] = __fadd2_rn(acc[(y >> 1) & 1], e);
              const __half2 h = __floats2half2_rn(e.x, e.y);
              w[16 * (k & 1) + (y >> 1)] = *reinterpret_cast<const uint32_t*>(&h);
            }
            if (k & 1) {
              tmem_st32(ts + 32 * (k - 1), w);
              tmem_stored();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.pfull[x][k >> 1]);
            }
          }
          acc[0] = __fadd2_rn(acc[0], acc[1]);
          l += acc[0].x + acc[0].y;
        } else if (lane == 0) {
          mbar_arrive(&sh.pfull[x][0]);
          mbar_arrive(&sh.pfull[x][1]);
        }
      }
      steps_done += (uint32_t)n;
      // (the next queries on their way to L2 while the sums are stored)
      more = take_next();
      if (more) {
        const Work& next = sh.now[x][(taken - 1) & 1];
        const __nv_bfloat16* const src =
            a.q + ((size_t)next.b * a.R * a.c.kv_heads * a.group + row_of(next)) * D;
#pragma unroll
        for (int k = 0; k < D; k += 64)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(src + k));
      }

      // the sums
      if (x < ops) wait_on(&sh.ofull[x][1], (count - 1) & 1, bad);
      tc_fence_after();
      float fac[2] = {1.f, 0.f};
      if (split) {
        sh.m[x][r] = x < ops ? mref : TV_NEG_INF;
        sh.l[x][r] = x < ops ? l : 0.f;
        tc_fence_before();                       // (each tile's threads read both tiles' sums)
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.merge);
        wait_on(&sh.merge, merged++ & 1, bad);
        tc_fence_after();
        const float m0 = sh.m[0][r], m1 = sh.m[1][r];
        mref = fmaxf(m0, m1);
        fac[0] = m0 == TV_NEG_INF ? 0.f : ex2(m0 - mref);
        fac[1] = m1 == TV_NEG_INF ? 0.f : ex2(m1 - mref);
        l = sh.l[0][r] * fac[0] + sh.l[1][r] * fac[1];
      }
      if (live) {
        const bool whole = p.whole();
        const float inv = !whole ? 1.f
                          : l == 0.f ? 0.f
                                     : pow2i(exponent_of(a.c, a.layer, 1, p.head)) / l;
        // the warp's first row among the CTA's pieces' rows, and its rows that there are
        const size_t part0 = (2 * (size_t)blockIdx.x + (p.s0 == 0)) * 2 * kTile +
                             (split ? 0 : x * kTile) + w0;
        const int rows = min(M - (m - lane), 32);
        fac[0] *= inv;
        fac[1] *= inv;
        // (split: of both tiles' sums half of the columns each)
        const int c0 = split ? x * (D / 2) : 0, c1 = split ? c0 + D / 2 : D;
        const uint32_t t0 = split ? tmem + 2 * kTile + lanes : to;
#pragma unroll 1
        for (int col = c0; col < c1; col += 32) {
          uint32_t c[32];
          tmem_ld32(t0 + col, c);
          tmem_wait(c);
#pragma unroll
          for (int y = 0; y < 32; ++y)
            c[y] = split && fac[0] == 0.f ? 0u : __float_as_uint(__uint_as_float(c[y]) * fac[0]);
          if (split && ops > 1) {
#pragma unroll
            for (int z = 0; z < 32; z += 16) {
              uint32_t d[16];
              tmem_ld16(t0 + D + col + z, d);
              tmem_wait16(d);
#pragma unroll
              for (int y = 0; y < 16; ++y)
                c[z + y] = __float_as_uint(__uint_as_float(c[z + y]) +
                                           (fac[1] == 0.f ? 0.f : __uint_as_float(d[y]) * fac[1]));
            }
          }
          if (whole) {
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              uint32_t w[4];
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const __nv_bfloat162 h =
                    __floats2bfloat162_rn(__uint_as_float(c[8 * z + 2 * y]),
                                          __uint_as_float(c[8 * z + 2 * y + 1]));
                w[y] = *reinterpret_cast<const uint32_t*>(&h);
              }
              sts128(piece_at(mine, r, col / 8 + z), w[0], w[1], w[2], w[3]);
            }
          } else {                               // 32 sums of a row, 8 lanes a row
#pragma unroll
            for (int z = 0; z < 8; ++z)
              sts128(piece_at(mine, r, z), c[4 * z], c[4 * z + 1], c[4 * z + 2], c[4 * z + 3]);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const int to_row = k + lane / 8;
              const uint4 v = lds128_at(piece_at(mine, w0 + to_row, lane % 8));
              if (to_row < rows)
                *reinterpret_cast<uint4*>(a.part + (part0 + to_row) * D + col + lane % 8 * 4) = v;
            }
            __syncwarp();
          }
        }
        if (whole) {
          __syncwarp();
          const int pieces = (c1 - c0) / 8, per = 32 / pieces, at = lane % pieces;
          uint4* const dst = reinterpret_cast<uint4*>(a.out) +
                             (size_t)p.b * a.R * a.c.kv_heads * a.group * (D / 8) + c0 / 8 + at;
          for (int k = 0; k < 32; k += per) {
            const int to_row = k + lane / pieces;
            const int from = __shfl_sync(0xffffffffu, row, to_row);
            const uint4 v = lds128_at(piece_at(mine, w0 + to_row, c0 / 8 + at));
            if (to_row < rows) dst[(size_t)from * (D / 8)] = v;
          }
          __syncwarp();
        }
        if (!whole && !(split && x == 1) && in)
          stats_of(a, D, gridDim.x)[part0 + lane] = make_float2(mref, l);
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

// Joins the pieces of an item that spans CTAs: block c * parts + part takes a part of the rows of
// the item that begins in CTA c and goes on in later ones.  Its factors first, for all rows and
// pieces at once, and then the sums with several pieces' loads on their way.
constexpr int kJoinRows = 16;

template <int D>
__global__ void __launch_bounds__(256) join_kernel(AttendArgs a, int split, int ctas) {
  extern __shared__ float join_fac[];                    // [pieces][kJoinRows]
  __shared__ float inv[kJoinRows];
  asm volatile("griddepcontrol.wait;" ::: "memory");     // (launched before the pieces are there)
  const int parts = (split ? kTile : 2 * kTile) / kJoinRows;
  const int c0 = blockIdx.x / parts, r0 = blockIdx.x % parts * kJoinRows, tid = threadIdx.x;
  const Split item = splits_of(a, D, ctas)[c0];
  if (item.b < 0) return;
  const int M = request_of(a, item.b).rows * a.group - item.m0;      // rows of the item
  if (r0 >= M) return;
  const int pieces = item.last - c0 + 1;
  auto row_of = [&](int k, int r) {
    return ((size_t)2 * (c0 + k) + (k == 0)) * 2 * kTile + r0 + r;
  };
  const float2* const stats = stats_of(a, D, ctas);
  // 16 neighbouring threads for a row
  const int r = tid / 16, sub = tid % 16;
  float top = TV_NEG_INF, sum = 0.f;
  if (r0 + r < M)
    for (int k = sub; k < pieces; k += 16) {
      const float2 ms = stats[row_of(k, r)];
      join_fac[k * kJoinRows + r] = ms.x;
      top = fmaxf(top, ms.x);
    }
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (r0 + r < M)
    for (int k = sub; k < pieces; k += 16) {
      const float m = join_fac[k * kJoinRows + r], part = stats[row_of(k, r)].y;
      const float f = part != part ? part : m == TV_NEG_INF ? 0.f : ex2(m - top);
      join_fac[k * kJoinRows + r] = f;
      sum += f * part;
    }
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (sub == 0) inv[r] = sum;
  __syncthreads();
  const float up = pow2i(exponent_of(a.c, a.layer, 1, item.head));
  for (int x = tid; x < kJoinRows * D / 4; x += 256) {
    const int row = x / (D / 4), col = x % (D / 4) * 4;
    if (r0 + row >= M) break;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = 0; k < pieces; ++k) {
      const float f = join_fac[k * kJoinRows + row];
      const float4 v = *reinterpret_cast<const float4*>(a.part + row_of(k, row) * D + col);
      y.x += f * v.x;
      y.y += f * v.y;
      y.z += f * v.z;
      y.w += f * v.w;
    }
    store_out(a, item.b, item.head, item.m0 + r0 + row, item.m0 + M, col, D, y, inv[row], up);
  }
}

template <int D>
int launch_tiles(const AttendArgs& a, int sm_count, cudaStream_t stream) {
  const size_t smem = (size_t)(2 + 2 * kStages) * kTile * D * 2 + 1024;
  static std::atomic<uint64_t> allowed{0};
  if (!allow_smem(tile_kernel<D>, smem, allowed)) return -5;
  const int split = (long long)a.R * a.group <= kTile;
  tile_kernel<D><<<sm_count, kTileThreads, smem, stream>>>(a, split);
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t join = {};
  join.gridDim = dim3((unsigned)(sm_count * ((split ? kTile : 2 * kTile) / kJoinRows)));
  join.blockDim = dim3(256);
  join.dynamicSmemBytes = (size_t)sm_count * kJoinRows * sizeof(float);
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
