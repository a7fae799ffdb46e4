// tv_attend.cu -- attention over the 4-bit key/value cache for few query rows per key/value
// head (sm_103a): decoding steps and small trees.
//
//   o_i = sum_j p_ij v_j,  p_i = softmax_j(scale q_i . k_j)  over the tokens j that row i sees.
//
// Bound by the cache's bytes, and next to that by the instructions that widen the codes.  One
// warp of a CTA copies whole pages of keys and values (they lie together) to a ring in shared
// memory by TMA, from piece to piece without a stop; eight take 16 tokens of a step each, and
// widen the codes in the registers of mma.sync fragments (tcgen05 wants its operands in shared
// memory: 4 bytes of traffic there per value, written and read, for the 9/16 that come from
// memory).  With lane = 4 g + t:
//   S^T [16 tokens x 8 rows]  = K Q^T      A: the lane's 2 tokens, g and g + 8, in 8 columns
//                                          (index t) of each 32; the order of columns inside
//                                          a product is free, so these are adjacent ones
//   O^T [16 columns x 8 rows] += V^T P^T   A: the lane's D / 8 columns of index g in its 4
//                                          tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9; codes of two
//                                          tokens are paired before they are widened
// and S^T's accumulators become P^T's operand by two 8 x 8 transposes.  Keys and values are
// exact in fp16, without the power of two of their head; queries are scaled by a power of
// two per row, so that their largest magnitude is in [2^14, 2^15), and rounded to fp16, which
// changes only columns 2^-21 below the row's largest and smaller.  Weights are 2^(t - m + 6) in
// fp16, rounded by at most 2^-12 of themselves: m is the largest t (log2(e) times the score) so
// far, or up to 8 below it, which saves most rescaling; they stay below 2^14 and keep all bits
// down to 2^-20 of the largest.  Sums are float32.
//
// Work is cut evenly: a step is 128 tokens (16 for each of 8 warps) of one item, an item is
// one (request, key/value head, tile of rows), and every CTA takes the same number of
// consecutive steps, found from the lengths on the device.  An item that spans CTAs is joined by
// the last of them to finish, in the order of its pieces.
//
// 128 requests of up to 8192 tokens, 8 heads of 128 columns, 4 query heads each: 211 to 218 us, 4.1
// to 4.3 TB/s of the cache (0.61 to 0.63 of what a copy reaches).  Nine warps twice an SM leave a
// thread 96 registers, and all three forms spill to local memory: 96 bytes stored and 208 loaded
// by a thread at 128 columns, 28 and 28 with 8 rows of 64, 144 and 280 with 16.  More rows go to
// the tiles of tv_attend_tile.cu (tv_launch_attend has both sides' times).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/tv.h"
#include "tv_attend.cuh"
#include "tv_cache.cuh"
#include "tv_device.cuh"
#include "tv_launch.h"
#include "tv_ptx.cuh"

namespace tvk {
namespace attend {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * (kWarps + 1);      // and the copying warp
constexpr int kUnit = 16;                        // tokens of a warp's step
static_assert(kStep == kUnit * kWarps, "a step is 16 tokens of each warp");
constexpr int kMaxRows = 16;                     // rows of an item, and so of a tree
constexpr int kPerSm = 2;

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

constexpr int kWorkSlots = 4;

// Steps that the ring holds, of 128 tokens' codes and scales, keys and values.
template <int D>
constexpr int kRing = D == 128 ? 3 : 6;
template <int D>
constexpr uint32_t kStepBytes = (uint32_t)kStep * D * 9 / 8;

__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t at) {
  uint16_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=h"(v) : "r"(at));
  return v;
}
__device__ __forceinline__ void consumers() {    // a barrier of the warps that do not copy
  asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
}

// Where a lane's codes and scales are in a step of the ring.
template <int D>
struct Lane {
  uint32_t k, ks, v, vs, plane;
  int page;                                      // of the step's
  __device__ __forceinline__ Lane(const CacheArgs& c, int warp, int lane) {
    const int g = lane >> 2, t = lane & 3;
    constexpr int kChunks = D / 32;
    const uint32_t block = (uint32_t)c.page_size * D * 9 / 16;
    const uint32_t slot = (uint32_t)(warp * kUnit) & (c.page_size - 1);
    page = (warp * kUnit) >> c.page_shift;
    plane = (uint32_t)c.page_size;               // tokens of a chunk's codes or scales
    const uint32_t keys = (uint32_t)page * 2 * block, values = keys + block;
    const uint32_t scales = plane * D / 2, chunk = (uint32_t)(g * kChunks / 8) * plane;
    k = keys + (slot + g) * 16 + t * 4;
    ks = keys + scales + (slot + g) * 2 + (t >> 1);
    v = values + (chunk + slot + 2 * t) * 16 + (g * (D / 16)) % 16;
    vs = values + scales + (chunk + slot + 2 * t) * 2;
  }
};
// Shared memory of a CTA; what follows it: the ring, and the warps' sums [kWarps][rows][D + 4].
struct alignas(16) Shared {
  uint64_t given[kWorkSlots], taken[kWorkSlots], full[8], empty[8];
  Piece pieces[kWorkSlots], now[2];              // the ring of them, and the consumers' two
  int more[kWorkSlots], going[2];
  uint32_t valid[8];                             // the pages of a step that are there
  Schedule plan;
  int last;
  float m[kWarps][kMaxRows], l[kWarps][kMaxRows];
  float fac[kWarps][kMaxRows], sum[kMaxRows], top[kMaxRows];
  int32_t parents[kMaxRows];
  uint32_t seen[kMaxRows];                       // bit j: an item's row sees the tree's row j
};

static_assert(sizeof(Shared) % 16 == 0, "the sums behind it are read 16 bytes at a time");

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, kPerSm) attend_kernel(AttendArgs a) {
  constexpr int kRows = 8 * NT;
  static_assert(kRows <= kMaxRows, "");
  constexpr int kDT = D / 16;                    // column tiles of O^T
  constexpr int kKS = D / 16;                    // products of S^T
  constexpr int kPitch = D + 4;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  const uint32_t ring = smem_u32(smem + sizeof(Shared));
  float* const sums =
      reinterpret_cast<float*>(smem + sizeof(Shared) + kRing<D> * (size_t)kStepBytes<D>);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int G = a.group, H = a.c.kv_heads;
  uint32_t bad = 0;

  if (tid == 0) {
    for (int i = 0; i < kWorkSlots; ++i) {
      mbar_init(&sh.given[i], 1);
      mbar_init(&sh.taken[i], 1);
    }
    for (int i = 0; i < kRing<D>; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], kWarps);
    }
    fence_mbar_init();
  }
  Walker walker;
  // (one row of 2000, 4000, 8000 tokens and 8 heads: 13.0, 18.4, 20.8 us with one step at least,
  // 11.8, 14.6, 17.3 with two, two and three.)
  const Shares shares = plan(a, sh.plan, kRows, blockIdx.x, gridDim.x, 4.f, walker);

  if (warp == kWarps) {
    // ---- pages to the ring ----
    const uint32_t block2 = (uint32_t)a.c.page_size * D * 9 / 8;      // keys and values
    const int pages = kStep >> a.c.page_shift;                        // of a step, 8 at most
    uint32_t count = 0;
    for (uint32_t n = 0;; ++n) {
      Piece& p = sh.pieces[n % kWorkSlots];
      if (lane == 0) {
        wait_on(&sh.taken[n % kWorkSlots], ((n / kWorkSlots) & 1) ^ 1, bad);
        sh.more[n % kWorkSlots] = bad ? -1 : walker.next(a, kRows, p);
        mbar_arrive(&sh.given[n % kWorkSlots]);
      }
      __syncwarp();
      if (sh.more[n % kWorkSlots] <= 0) break;
      const int b = p.b, s0 = p.s0, s1 = p.s1, tokens = p.tokens;
      const uint8_t* const blocks =
          a.c.data + ((size_t)a.layer * a.c.pages * H + p.head) * block2;
      const int32_t* const table = a.t.table + (size_t)b * a.t.max_pages;
      auto page_at = [&](int s) -> int {
        const int pos = s * kStep + (lane << a.c.page_shift);
        return lane < pages && s < s1 && pos < tokens
                   ? __ldg(table + (pos >> a.c.page_shift))            // (inside the table)
                   : -2;
      };
      int page = page_at(s0), page_next = page_at(s0 + 1);
      for (int s = s0; s < s1; ++s, ++count) {
        const uint32_t stage = count % kRing<D>;
        bool there = (unsigned)page < (unsigned)a.c.pages;
        if (!there && page != -2) atomicOr(a.status, (uint32_t)TV_STATUS_BAD_PAGE);
        wait_on(&sh.empty[stage], ((count / kRing<D>) & 1) ^ 1, bad);
        const bool gave_up = __any_sync(0xffffffffu, bad != 0);
        there = there && !gave_up;               // (copied to what is free only)
        const uint32_t valid = __ballot_sync(0xffffffffu, there);
        if (lane == 0) {
          sh.valid[stage] = valid;
          mbar_arrive_expect_tx(&sh.full[stage], (uint32_t)__popc(valid) * block2);
        }
        __syncwarp();
        if (there)
          tma_load_1d(smem + sizeof(Shared) + stage * (size_t)kStepBytes<D> + lane * block2,
                      blocks + (size_t)page * H * block2, block2, &sh.full[stage]);
        page = page_next;
        page_next = page_at(s + 2);
      }
    }
    zero_rows(a, D, blockIdx.x, gridDim.x);
    // (no copy is on its way when the CTA ends, although a warp that gave up may not have waited)
    for (uint32_t i = count - min(count, (uint32_t)kRing<D>); i < count; ++i)
      if (!mbar_wait(&sh.full[i % kRing<D>], (i / kRing<D>) & 1)) bad = 1;
    if (bad && lane == 0) atomicOr(a.status, (uint32_t)TV_STATUS_TIMEOUT);
    return;
  }

  const Lane<D> at(a.c, warp, lane);
  uint32_t count = 0, n = 0;
  for (;; ++n) {
    if (tid == 0) {                              // (the others meet at barriers)
      wait_on(&sh.given[n % kWorkSlots], (n / kWorkSlots) & 1, bad);
      if (sh.more[n % kWorkSlots] < 0) bad = 1;
      sh.going[n & 1] = !bad && sh.more[n % kWorkSlots] > 0;
      sh.now[n & 1] = sh.pieces[n % kWorkSlots];
      mbar_arrive(&sh.taken[n % kWorkSlots]);
    }
    consumers();
    if (!sh.going[n & 1]) break;
    const Piece& p = sh.now[n & 1];
    const int b = p.b, head = p.head, m0 = p.m0, s0 = p.s0, s1 = p.s1;
    const int len = p.rq.len, nrows = p.rq.rows, tokens = p.tokens;
    const bool masked = (long long)s1 * kStep > len;       // some tokens are the tree's
    if (masked && a.parents) {
      if (tid < nrows) sh.parents[tid] = a.parents[(size_t)b * a.R + tid];
      consumers();
      if (tid < kRows) {
        uint32_t seen = 0;
        if (m0 + tid < nrows * G &&
            !walk(sh.parents, (m0 + tid) / G, [&](int j) { seen |= 1u << j; }))
          atomicOr(a.status, (uint32_t)TV_STATUS_BAD_TREE);
        sh.seen[tid] = seen;
      }
      consumers();
    }

    // queries: row 8 n + g, the columns of index t, in the order of a product's pairs
    uint32_t q[NT][kKS][2];
    float fac[NT][2];                            // of rows 8 n + 2 t and the next
    const int ek = exponent_of(a.c, a.layer, 0, head), ev = exponent_of(a.c, a.layer, 1, head);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int m = m0 + 8 * n + g;
      const bool in = m < nrows * G;
      const uint4* const src = reinterpret_cast<const uint4*>(
          a.q + (((size_t)b * a.R + (in ? m / G : 0)) * H * G + (size_t)head * G + m % G) * D +
          t * 8);
      uint32_t w[D / 8];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const uint4 u = in ? __ldg(src + 4 * i) : make_uint4(0, 0, 0, 0);
        w[4 * i] = u.x;
        w[4 * i + 1] = u.y;
        w[4 * i + 2] = u.z;
        w[4 * i + 3] = u.w;
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
        top = max_nan(top, max_nan(fabsf(bf16_lo(w[i])), fabsf(bf16_hi(w[i]))));
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const QueryScale s(top);
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
        q[n][i >> 1][i & 1] = pack_half2(s.apply(bf16_lo(w[i])), s.apply(bf16_hi(w[i])));
      const float f = s.factor(a.scale_log2e, ek);
      fac[n][0] = __shfl_sync(0xffffffffu, f, 8 * t);
      fac[n][1] = __shfl_sync(0xffffffffu, f, 8 * t + 4);
    }

    float o[NT][kDT][4], mref[NT][2], l[NT][2], off[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < kDT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[n][i][k] = 0.f;
      mref[n][0] = mref[n][1] = TV_NEG_INF;
      l[n][0] = l[n][1] = 0.f;
      off[n][0] = off[n][1] = kLift;
    }

    for (int s = s0; s < s1; ++s, ++count) {
      const int pos = s * kStep + warp * kUnit;
      const uint32_t stage = count % kRing<D>;
      wait_on(&sh.full[stage], (count / kRing<D>) & 1, bad);
      const bool there = sh.valid[stage] >> at.page & 1;
      if (!there) {
        __syncwarp();                            // (all lanes have read which pages there are)
        if (lane == 0) mbar_arrive(&sh.empty[stage]);
        continue;
      }
      const uint32_t step = ring + stage * kStepBytes<D>;
      // S^T
      float st[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) st[n][k] = 0.f;
      {
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {                 // 8 columns: two products
          uint32_t h[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            decode8(lds32(step + at.k + w * at.plane * 16 + 128 * i), h[i]);
            const uint32_t s2 = decode_scales(
                __byte_perm(lds8(step + at.ks + w * at.plane * 2 + 16 * i), 0u, 0x4400u));
#pragma unroll
            for (int k = 0; k < 4; ++k) h[i][k] = mul2(h[i][k], s2);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t af[4] = {h[0][2 * k], h[1][2 * k], h[0][2 * k + 1], h[1][2 * k + 1]};
#pragma unroll
            for (int n = 0; n < NT; ++n)
              mma16816(st[n], af, q[n][2 * w + k][0], q[n][2 * w + k][1]);
          }
        }
      }

      // the values' codes, and the step is this warp's no longer
      constexpr int kV = D / 64;                 // words of a lane's D / 8 columns of a token
      uint32_t v[4][kV], vs[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {              // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        const uint32_t from = step + at.v + ((i & 1) + 8 * (i >> 1)) * 16;
        if constexpr (D == 128) {
          const uint2 u = lds64(from);
          v[i][0] = u.x;
          v[i][1] = u.y;
        } else {
          v[i][0] = lds32(from);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) vs[i] = lds32(step + at.vs + 16 * i);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.empty[stage]);

      // weights: st[n][k] is token g (k < 2) or g + 8, row 8 n + 2 t + (k & 1)
      bool grow = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float x = st[n][k] * fac[n][k & 1];
          if (pos + kUnit > len) {
            const int at = pos + g + (k & 2) * 4 - len, row = 8 * n + 2 * t + (k & 1);
            bool on = at < 0;
            if (!on && at < nrows && at + len < tokens)
              on = a.parents ? (sh.seen[row] >> at & 1u) != 0u : at <= (m0 + row) / G;
            x = on ? x : TV_NEG_INF;
          }
          st[n][k] = x;
          grow = grow || x > mref[n][k & 1] + kSlack;
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float top = fmaxf(st[n][k], st[n][k + 2]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            if (top > mref[n][k]) {
              const float down = ex2(mref[n][k] - top);    // (0 from -inf)
              mref[n][k] = top;
              off[n][k] = kLift - top;
              l[n][k] *= down;
#pragma unroll
              for (int i = 0; i < kDT; ++i) {
                o[n][i][k] *= down;
                o[n][i][k + 2] *= down;
              }
            }
          }
      }
      uint32_t pb[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = ex2(st[n][k] + off[n][k & 1]);
          l[n][k & 1] += x[k];
        }
        pb[n][0] = transpose8(pack_half2(x[0], x[1]));
        pb[n][1] = transpose8(pack_half2(x[2], x[3]));
      }

      // O^T
      {
        uint32_t sc[2];                                    // of tokens 2 t, 2 t + 1; 8 further
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool upper = D == 128 ? (g & 1) : (g & 2);
          uint32_t two = __byte_perm(vs[i], 0u, upper ? 0x4431u : 0x4420u);
          // (bytes behind the last token may be anything, a NaN among it)
          const int left = tokens - (pos + 2 * t + 8 * i);
          if (left < 2) two = left < 1 ? 0u : two & 0xffu;
          sc[i] = decode_scales(two);
        }
#pragma unroll
        for (int w = 0; w < kV; ++w) {                     // 8 columns: four tiles
          uint32_t e[2][4], f[2][4];                       // even and odd columns, token pairs
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t x = v[2 * i][w], y = v[2 * i + 1][w];
            decode8((x & 0x0f0f0f0fu) | (y << 4 & 0xf0f0f0f0u), e[i]);
            decode8((x >> 4 & 0x0f0f0f0fu) | (y & 0xf0f0f0f0u), f[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              e[i][k] = mul2(e[i][k], sc[i]);
              f[i][k] = mul2(f[i][k], sc[i]);
            }
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t af[4] = {e[0][k], f[0][k], e[1][k], f[1][k]};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816(o[n][4 * w + k], af, pb[n][0], pb[n][1]);
          }
        }
      }
    }

    // the warps' sums joined.  o[n][i][k]: column (D / 8) g + 2 i + (k >> 1), row
    // 8 n + 2 t + (k & 1)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[n][k] += __shfl_xor_sync(0xffffffffu, l[n][k], x);
        const int row = 8 * n + 2 * t + k;
        if (g == 0) {
          sh.m[warp][row] = mref[n][k];
          sh.l[warp][row] = l[n][k];
        }
        float* const dst = sums + ((size_t)warp * kRows + row) * kPitch + g * (D / 8);
#pragma unroll
        for (int i = 0; i < kDT; ++i)
          *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(o[n][i][k], o[n][i][k + 2]);
      }
    consumers();
    if (tid < kRows) {
      float top = TV_NEG_INF, sum = 0.f;
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.m[w][tid]);
      for (int w = 0; w < kWarps; ++w) {
        const float f = sh.m[w][tid] == TV_NEG_INF ? 0.f : ex2(sh.m[w][tid] - top);
        // (a row that is not a number has no maximum, and its sums are NaN)
        sh.fac[w][tid] = sh.l[w][tid] != sh.l[w][tid] ? sh.l[w][tid] : f;
        sum += sh.l[w][tid] * sh.fac[w][tid];
      }
      sh.top[tid] = top;
      sh.sum[tid] = sum;
    }
    consumers();
    const bool whole = p.whole();
    const float up = pow2i(ev);
    const int slot = 2 * (int)blockIdx.x + (s0 == 0);
    for (int x = tid; x < kRows * D / 4; x += 32 * kWarps) {
      const int row = x / (D / 4), col = x % (D / 4) * 4;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < kWarps; ++w) {
        const float4 v =
            *reinterpret_cast<const float4*>(sums + ((size_t)w * kRows + row) * kPitch + col);
        const float f = sh.fac[w][row];
        y.x += f * v.x;
        y.y += f * v.y;
        y.z += f * v.z;
        y.w += f * v.w;
      }
      if (whole)
        store_out(a, b, head, m0 + row, nrows * G, col, D, y, sh.sum[row], up);
      else
        reinterpret_cast<float4*>(a.part)[(size_t)slot * (kRows * D / 4) + x] = y;
    }
    if (!whole) {
      float2* const stats = reinterpret_cast<float2*>(a.part + (size_t)2 * gridDim.x * kRows * D);
      if (tid < kRows) stats[(size_t)slot * kRows + tid] = make_float2(sh.top[tid], sh.sum[tid]);
      // pieces lie in the CTAs from the one with the item's first step to that with its last
      const int c0 = shares.owner(p.first), c1 = shares.owner(p.first + p.steps - 1);
      __threadfence();
      consumers();
      if (tid == 0) {
        const int seen = atomicAdd(&a.counters[c0], 1);
        sh.last = seen == c1 - c0;
        if (sh.last) a.counters[c0] = 0;
      }
      consumers();
      if (sh.last) {
        __threadfence();
        for (int x = tid; x < kRows * D / 4; x += 32 * kWarps) {
          const int row = x / (D / 4), col = x % (D / 4) * 4;
          float top = TV_NEG_INF, sum = 0.f;
#pragma unroll 8
          for (int c = c0; c <= c1; ++c)
            top = fmaxf(top, __ldcg(&stats[(size_t)(2 * c + (c == c0)) * kRows + row]).x);
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const size_t at = 2 * c + (c == c0);
            const float2 ms = __ldcg(&stats[at * kRows + row]);
            const float f = ms.y != ms.y ? ms.y : ms.x == TV_NEG_INF ? 0.f : ex2(ms.x - top);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part) +
                                    at * (kRows * D / 4) + x);
            sum += f * ms.y;
            y.x += f * v.x;
            y.y += f * v.y;
            y.z += f * v.z;
            y.w += f * v.w;
          }
          store_out(a, b, head, m0 + row, nrows * G, col, D, y, sum, up);
        }
      }
    }
    consumers();
  }
  // after a wait that gave up the pieces that are left arrive all the same, so that the counters
  // are 0 for the next call
  if (bad && tid == 0 && (long long)blockIdx.x < shares.ctas) {
    Walker w = {sh.plan.request, sh.plan.offset, shares.begin(blockIdx.x),
                shares.begin(blockIdx.x + 1)};
    Piece p;
    for (uint32_t i = 0; w.next(a, kRows, p); ++i) {
      if (i < n || p.whole()) continue;
      const int c0 = shares.owner(p.first), c1 = shares.owner(p.first + p.steps - 1);
      if (atomicAdd(&a.counters[c0], 1) == c1 - c0) a.counters[c0] = 0;
    }
  }
  if (bad && lane == 0) atomicOr(a.status, (uint32_t)TV_STATUS_TIMEOUT);
}

template <int D, int NT>
int launch(const AttendArgs& a, int sm_count, cudaStream_t stream) {
  const size_t smem = sizeof(Shared) + kRing<D> * (size_t)kStepBytes<D> +
                      (size_t)kWarps * 8 * NT * (D + 4) * sizeof(float);
  static std::atomic<uint64_t> allowed{0};
  if (!allow_smem(attend_kernel<D, NT>, smem, allowed)) return -5;
  attend_kernel<D, NT><<<kPerSm * sm_count, kThreads, smem, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

}  // namespace attend
}  // namespace tvk

using namespace tvk::attend;

size_t tv_attend_scratch(int sm_count) {
  // two pieces of each CTA, of 16 rows of 64 columns or 8 of 128 (and their statistics)
  const size_t few =
      (size_t)kPerSm * sm_count * 2 * (kMaxRows * 64 + 2 * kMaxRows) * sizeof(float);
  return std::max(few, tv_attend_tile_scratch(sm_count));
}
int tv_attend_counters(int sm_count) { return kPerSm * sm_count; }

// Times in us by warps and on the tiles (8 heads, pages of 64; 1 x 2000 is one request of 2000
// tokens, 32 x 1000 are requests of 500 to 1000, 128 x 4096 of 2048 to 4096), rows as query heads
// of one token; a tree's rows take up to 3 % more by warps, on the tiles up to 8 % (37 % at 64
// columns).  9 rows and more of 128 columns, and 24 and 32 of 64, were timed by warps in forms that
// are not kept.  The rule's worst place is one short request of 9 to 16 rows of 128 columns.
//                  rows     1 x 2000    1 x 131000    32 x 1000    128 x 4096
//     128 columns   1, 4     11   18       51   81        23   38     119  232
//                   8        12   18       51   81        23   40     120  233
//                   9, 16    18   22      165   87        59   41     403  238
//      64 columns   4, 8     11   15       38   59        19   31      82  183
//                   9, 16    13   15       50   60        25   32     126  185
//                  24, 32    22   15      218   61        77   32     630  188
int tv_launch_attend(const AttendArgs& a, int sm_count, cudaStream_t stream) {
  const long long rows = (long long)a.R * a.group;
  const int most = a.c.head_dim == 128 ? 8 : kMaxRows;
  if (rows > most) return tv_launch_attend_tile(a, sm_count, stream);
  if (a.c.head_dim == 128) return launch<128, 1>(a, sm_count, stream);
  return rows <= 8 ? launch<64, 1>(a, sm_count, stream) : launch<64, 2>(a, sm_count, stream);
}
