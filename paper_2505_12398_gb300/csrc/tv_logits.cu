// tv_logits.cu -- penalties, biases and grammar masks on the target's logits, per tree
// row, with the row normalisers that verification takes (sm_103a).
//
// Row i of a request's tree predicts the token after node i, so the text it has seen is
// the request's own and the drafted tokens on the path from the root to node i.  For
// token x with n = (times generated) + (times on that path), in 32 bits:
//   l1 = l > 0 ? l / rep : l * rep     where x is in the prompt or n > 0
//   l2 = (l1 - freq n) - pres          where n > 0
//   l3 = l2 + bias[x]
//   l4 = -inf                          where the row's grammar mask has x's bit at 0
// rounded once to the logits' type, and (max, sum 2^((l4 - max) c)) of what is stored.
//
// A request's context is what its text adds up to: per token the count of generated
// occurrences and a prompt bit in one word, a bias, and one bit in a bitmap of the
// tokens that have any of them.  Those are a few in a hundred, so the bitmap (1/16 of
// the logits' bytes) is all that is read for the others.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "tv_device.cuh"
#include "tv_launch.h"
#include "tv_ptx.cuh"

namespace tvk {
namespace logits {

constexpr int kSegment = 65536;         // tokens whose bits are in shared memory at a time
constexpr int kPathBits = 4096;
constexpr int kListed = 96;              // marked tokens of a warp's step that it shares out
constexpr int kMaxCluster = 8;
constexpr uint32_t kBadTree = 1u, kBadToken = 2u, kBadSlot = 256u, kBadMask = 512u;

// A block of 8 logits, and how many blocks a thread has on its way (64 bytes).
template <typename L> struct Block;
template <> struct Block<Bf16Logits> {
  using elem = __nv_bfloat16;
  static constexpr int kBlocks = 4, kWords = 4;
};
template <> struct Block<F32Logits> {
  using elem = float;
  static constexpr int kBlocks = 2, kWords = 8;
};

__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float get(const float* p) { return *p; }

// The logits may be processed in place, so that they are not read-only for the kernel.
__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}
__device__ __forceinline__ void st16(void* p, const uint32_t* w) {
  asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]),
               "r"(w[2]), "r"(w[3])
               : "memory");
}

struct Row {
  const uint32_t* counts;   // of the request's slot, or nullptr
  const float* bias;
  float rep, inv_rep, freq, pres;
};

// l / rep for l > 0, with inv = 1 / rep: the product with inv and one step of Newton's
// iteration on its residual (P. Markstein, Computation of elementary functions on the IBM RISC
// System/6000 processor, IBM J. Res. Dev. 34, 1990).  The residual is exact short of underflow,
// and the step leaves 2^-24 of its own size, so that the result is the nearest float32 unless
// the quotient is within 2^-23 of a unit of the middle of two.  Where the residual is no number
// (a quotient that overflows, an infinite l) the product stands.  With it, with the product
// alone (one more rounding), and with the compiler's division, which spills: 737, 735 and 777
// us at 128 x 61 x 128256 in bf16, 69.7, 68.6 and 74.6 at 32 x 27 x 32003 in fp32; where nearly
// all tokens are marked (500 x 61 x 1003, bf16) 232 and 225.
__device__ __forceinline__ float quotient(float l, float rep, float inv) {
  const float q = __fmul_rn(l, inv), e = fmaf(-q, rep, l);
  return fabsf(e) < -TV_NEG_INF ? fmaf(e, inv, q) : q;
}

// The logit of a marked token, on the path `times` times.
__device__ __forceinline__ float penalised(float l, uint32_t count, float bias, uint32_t times,
                                           const Row& r) {
  const uint32_t n = (count >> 1) + times;
  if (n > 0 || (count & 1u)) l = l > 0.f ? quotient(l, r.rep, r.inv_rep) : __fmul_rn(l, r.rep);
  if (n > 0) l = __fsub_rn(__fsub_rn(l, __fmul_rn(r.freq, (float)n)), r.pres);
  return __fadd_rn(l, bias);
}

// Blocks outside the allowed bits become -inf.  bf16: four bits at a time, each first to
// the sign of a byte of its own (their products with 2^7, 2^14, 2^21 and 2^28 do not
// overlap), the signs then through the bytes of two words.
__device__ __forceinline__ void mask_block(uint32_t (&w)[4], uint32_t allowed) {
#pragma unroll
  for (int k = 0; k < 4; k += 2) {
    const uint32_t signs = (allowed >> (2 * k) & 0xfu) * 0x10204080u;
    uint32_t lo, hi;
    asm("prmt.b32 %0, %1, %1, 0x9988;" : "=r"(lo) : "r"(signs));
    asm("prmt.b32 %0, %1, %1, 0xbbaa;" : "=r"(hi) : "r"(signs));
    w[k] = (w[k] & lo) | (0xff80ff80u & ~lo);
    w[k + 1] = (w[k + 1] & hi) | (0xff80ff80u & ~hi);
  }
}
__device__ __forceinline__ void mask_block(uint32_t (&w)[8], uint32_t allowed) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (!(allowed >> k & 1u)) w[k] = 0xff800000u;
}

// The larger value; kNan: NaN if either is, else the other one.
template <bool kNan>
__device__ __forceinline__ float max_of(float a, float b) {
  if constexpr (!kNan) return fmaxf(a, b);
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// The i-th pair of logits of a thread's blocks, and the largest of all.
template <int N>
__device__ __forceinline__ float2 pair_of(const uint32_t (&w)[N][4], int i) {
  const uint32_t u = w[i >> 2][i & 3];
  return make_float2(bf16_lo(u), bf16_hi(u));
}
template <int N>
__device__ __forceinline__ float2 pair_of(const uint32_t (&w)[N][8], int i) {
  return make_float2(__uint_as_float(w[i >> 2][2 * (i & 3)]),
                     __uint_as_float(w[i >> 2][2 * (i & 3) + 1]));
}
template <bool kNan, int N>
__device__ __forceinline__ float largest(const uint32_t (&w)[N][4]) {
  __nv_bfloat162 hm = *reinterpret_cast<const __nv_bfloat162*>(&w[0][0]);
#pragma unroll
  for (int i = 1; i < 4 * N; ++i) {
    const __nv_bfloat162 h = *reinterpret_cast<const __nv_bfloat162*>(&w[i >> 2][i & 3]);
    hm = kNan ? __hmax2_nan(hm, h) : __hmax2(hm, h);
  }
  return max_of<kNan>(__low2float(hm), __high2float(hm));
}
template <bool kNan, int N>
__device__ __forceinline__ float largest(const uint32_t (&w)[N][8]) {
  float m = __uint_as_float(w[0][0]);
#pragma unroll
  for (int i = 1; i < 8 * N; ++i) m = max_of<kNan>(m, __uint_as_float(w[i >> 3][i & 7]));
  return m;
}

__device__ __forceinline__ float rescale(const Bf16Logits&, float v, float m, float2 ch,
                                         float2 cl);
__device__ __forceinline__ float rescale(const F32Logits&, float v, float m, float2 ch,
                                         float2 cl);

// What m c = m (ch + cl) leaves beside the rounding of m ch to fp32.
__device__ __forceinline__ float beside(float m, float ch, float cl) {
  return fmaf(m, ch, -__fmul_rn(m, ch)) + m * cl;
}
// A thread's running sum, between the form in which it is kept where |m| < far (below) and
// the sum of 2^((v - m) c).
__device__ __forceinline__ float kept(float s, float m, float ch, float cl, float far) {
  return fabsf(m) < far ? s * ex2(beside(m, ch, cl)) : s;
}
__device__ __forceinline__ float settled(float s, float m, float ch, float cl, float far) {
  return fabsf(m) < far ? s * ex2(-beside(m, ch, cl)) : s;
}

// Adds blocks to a thread's running (max, sum).  Kept is the sum of 2^(v c - round(max ch)):
// two multiply-adds and one exponential a logit; what the rounding left of max c is put
// right once at the end.  A weight is then off by the two roundings of its exponent, within
// 2^-23 |(v - max) c| ln 2 to either side: of a sum, whose weights lie at 2^0 to 2^-17 of the
// largest for the most part, below 1.4e-6 at the very worst and 1e-7 as it goes.  (Without
// the product with cl all weights would be off to the same side.)  Blocks with a NaN (which
// weighs nothing) or with a maximum too far out for the product (|max| >= far = 2^20 / ch)
// are summed from exact differences instead; those, and a maximum with 0 for every logit,
// took 8 us more at 128 x 61 x 128256 in bf16.
template <typename L, int N, int W>
__device__ __forceinline__ void add_blocks(const uint32_t (&w)[N][W], float2 ch, float2 cl,
                                           float far, float& m_run, float& s_run) {
  const float m = largest<true>(w);
  if (m == TV_NEG_INF) return;           // (all masked)
  float2 acc[4];
  if (fabsf(m) < far && (fabsf(m_run) < far || m_run == TV_NEG_INF)) {
    if (m > m_run) {
      if (m_run != TV_NEG_INF) s_run *= ex2(__fmul_rn(m_run, ch.x) - __fmul_rn(m, ch.x));
      m_run = m;
    }
    const float mc = __fmul_rn(m_run, ch.x);
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      const float2 v = pair_of(w, i);      // (-inf: cl > 0, so that no infinities cancel)
      const float2 x = __ffma2_rn(v, cl, __ffma2_rn(v, ch, make_float2(-mc, -mc)));
      const float2 e = make_float2(ex2(x.x), ex2(x.y));
      acc[i & 3] = i < 4 ? e : __fadd2_rn(acc[i & 3], e);
    }
  } else {
    const float finite = largest<false>(w);
    s_run = settled(s_run, m_run, ch.x, cl.x, far);
    if (finite > m_run) {
      if (m_run != TV_NEG_INF) s_run *= rescale(L(), m_run, finite, ch, cl);
      m_run = finite;
    }
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      const float2 d = __fadd2_rn(pair_of(w, i), make_float2(-m_run, -m_run));
      const float2 x = __ffma2_rn(d, ch, __fmul2_rn(d, cl));
      // (-inf and NaN weigh nothing, at any temperature)
      const float2 e = make_float2(fmaxf(ex2(x.x), 0.f), fmaxf(ex2(x.y), 0.f));
      acc[i & 3] = i < 4 ? e : __fadd2_rn(acc[i & 3], e);
    }
    s_run = kept(s_run, m_run, ch.x, cl.x, far);
    const float k = kept(1.f, m_run, ch.x, cl.x, far);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = __fmul2_rn(acc[i], make_float2(k, k));
  }
  const float2 s2 = __fadd2_rn(__fadd2_rn(acc[0], acc[1]), __fadd2_rn(acc[2], acc[3]));
  s_run += s2.x + s2.y;
}

__device__ __forceinline__ float rescale(const Bf16Logits&, float v, float m, float2 ch,
                                         float2 cl) {
  return exp2_split(v - m, 0.f, ch.x, cl.x);
}
__device__ __forceinline__ float rescale(const F32Logits&, float v, float m, float2 ch,
                                         float2 cl) {
  return F32Logits::exp_rel(v, m, ch.x, cl.x);
}

// Adds one logit to a running (max, sum).
template <typename L>
__device__ __forceinline__ void add_one(const L&, float v, float2 ch, float2 cl, float& m_run,
                                        float& s_run) {
  if (v > m_run) {
    s_run = 1.f + (m_run == TV_NEG_INF ? 0.f : s_run * rescale(L(), m_run, v, ch, cl));
    m_run = v;
  } else if (m_run != TV_NEG_INF) {
    s_run += rescale(L(), v, m_run, ch, cl);
  }
}

// 32 bits of a bitmap row of `words` words from bit 32 w - shift on (bits before the row
// and past it are 0).
__device__ __forceinline__ uint32_t shifted(const uint32_t* row, int words, long long w,
                                            int shift) {
  const uint32_t hi = w < words ? row[w] : 0u;
  if (shift == 0) return hi;
  const uint32_t lo = w > 0 && w - 1 < words ? row[w - 1] : 0u;
  return __funnelshift_r(lo, hi, 32 - shift);
}

// One cluster of CTAs per row.  What bounds it: the logits' bytes, read and written once,
// with the loads of the next step on their way while this one is worked on, and the marked
// tokens, whose counts and biases are gathered in 32-byte sectors and put through shared
// memory.  At 128 x 61 x 128256 in bf16, 1 in 100 tokens marked, 737 us, 5.5 TB/s (some 95 us
// less with none marked; 600 at the copy's rate); at 32 x 27 x 32003 in fp32, rows that start at
// any element and 1 in 7 tokens marked, 69.5 us, 3.2 TB/s (49 with none, 33); one row of 128256
// takes 5.8 us in bf16 and 7.6 in fp32, one after the other, on a cluster of 8 CTAs, most of it
// the launch, the look-ups and the join.  The 64 registers a thread that four CTAs of 256 leave
// are all used: the fp32 forms and the bf16 form of 128 threads spill 20 to 56 bytes.
//
// A row is taken in blocks of 8 logits at 8-element
// boundaries of the whole array (16-byte loads wherever the row starts; the first and last
// block may hold elements of other rows, which are neither read nor written): position p
// of a row is its token p - off.  Shared memory holds two bytes for each block: a bit for
// each token that the grammar and the row's ends leave, and for each of those that has a
// count, a bias or a place on the path; only their counts and biases are gathered.
// Tried and slower at 128 x 61 x 128256: bits of 131072 tokens at a time (833 us for then 752),
// the row's marked tokens listed beforehand (1152), loads by a warp of their own through
// shared memory with persistent CTAs (1502).
template <typename L, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
    process_kernel(ProcessArgs a) {
  using E = typename Block<L>::elem;
  constexpr int NB = Block<L>::kBlocks, W = Block<L>::kWords;
  extern __shared__ __align__(16) uint32_t dyn[];
  __shared__ int n_path_s;
  __shared__ uint32_t path_bits[kPathBits / 32];     // (the path's tokens, modulo kPathBits)
  __shared__ float red[2][kThreads / 32];
  __shared__ float2 joined[kMaxCluster];
  const int R = a.N + 1, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  uint4* stage = reinterpret_cast<uint4*>(dyn);                    // [NB * W / 4][kThreads]
  uint16_t* bits = reinterpret_cast<uint16_t*>(dyn + NB * W * kThreads);   // [kSegment / 8]
  uint16_t* lists = bits + kSegment / 8;                           // [kThreads / 32][2][kListed]
  int* path = reinterpret_cast<int*>(lists + kThreads / 32 * 2 * kListed);   // [R], the tree's
  int* par = path + R;                                             // parents and tokens
  int* tok = par + R;
  uint32_t C, rank;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  // (the CTAs write to the first one's shared memory at the end, by when it has to run)
  if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const int row_id = blockIdx.x / C, b = row_id / R, node = row_id - b * R;
  const size_t row = row_id, start = row * a.V;
  const int off = (int)(start & 7);
  const int words = (a.V + 31) / 32;
  uint32_t found = 0;

  // this CTA's positions [p_lo, p_hi), whole steps of the block, and its whole blocks [lo,
  // hi) (what is left at the row's ends is taken element by element at the end)
  constexpr int kBlocks = NB * kThreads, kStep = 8 * kBlocks;
  const long long positions = (long long)a.V + off;
  const long long steps = (positions + kStep - 1) / kStep, per = (steps + C - 1) / C;
  const long long p_lo = min(positions, rank * per * kStep);
  const long long p_hi = min(positions, p_lo + per * kStep);
  const int lo = p_lo == 0 && off > 0 ? 1 : 0, hi = (int)((p_hi - p_lo) / 8);
  const int blocks = (hi + kBlocks - 1) / kBlocks * kBlocks;
  const E* const in = static_cast<const E*>(a.logits) + (start - off + p_lo) + 8 * tid;
  E* const out = static_cast<E*>(a.out) + (start - off + p_lo) + 8 * tid;
  const int x0 = (int)(p_lo - off) + 8 * tid;      // the token at this thread's first position
  // the first step's logits are on their way while all of the rest is looked up
  uint32_t next[NB][W];
  auto fetch = [&](int b0) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int blk = b0 + tid + j * kThreads;
      if (blk >= lo && blk < hi) {
#pragma unroll
        for (int k = 0; k < W; k += 4) {
          const uint4 u = ld16(reinterpret_cast<const char*>(in + 8 * b0) +
                               j * kThreads * 8 * (int)sizeof(E) + 4 * k);
          next[j][k] = u.x;
          next[j][k + 1] = u.y;
          next[j][k + 2] = u.z;
          next[j][k + 3] = u.w;
        }
      }
    }
  };
  fetch(0);

  // the request, and the tree for the drafted path to this row
  int slot = a.slots ? a.slots[b] : b;
  int mi = a.mask_index ? a.mask_index[row] : -1;
  if (node > 0) {
    for (int k = tid; k < node + 1; k += kThreads) {
      par[k] = a.parents[(size_t)b * R + k];
      tok[k] = a.tokens[(size_t)b * R + k];
    }
  }
  Row r;
  r.rep = a.penalties ? a.penalties[3 * b] : 1.f;
  r.inv_rep = 1.f / r.rep;
  r.freq = a.penalties ? a.penalties[3 * b + 1] : 0.f;
  r.pres = a.penalties ? a.penalties[3 * b + 2] : 0.f;
  if (a.counts && (slot < 0 || slot >= a.n_slots)) {
    found |= kBadSlot;
    slot = -1;
  }
  r.counts = a.counts && slot >= 0 ? a.counts + (size_t)slot * a.V : nullptr;
  r.bias = r.counts ? a.bias + (size_t)slot * a.V : nullptr;
  const uint32_t* marks = r.counts ? a.marks + (size_t)slot * words : nullptr;
  if (mi < -1 || mi >= a.n_masks) {
    found |= kBadMask;
    mi = -1;
  }
  const uint32_t* grammar = mi >= 0 ? a.masks + (size_t)mi * words : nullptr;
  // a byte of allowed and one of marked tokens for each block of a segment
  auto look_up = [&](int seg) {
    const int n = min(kSegment / 8, blocks - seg) / 4;
    for (int w = tid; w < n; w += kThreads) {
      const long long at = (p_lo + 8ll * seg) / 32 + w;
      uint32_t ok = grammar ? shifted(grammar, words, at, off) : 0xffffffffu;
      if (seg == 0 && w == 0 && lo) ok &= 0xffffff00u;
      const int left = 8 * (hi - seg) - 32 * w;
      if (left < 32) ok &= left > 0 ? (1u << left) - 1u : 0u;
      const uint32_t mk = marks ? shifted(marks, words, at, off) & ok : 0u;
      reinterpret_cast<uint2*>(bits)[w] =
          make_uint2(__byte_perm(ok, mk, 0x5140), __byte_perm(ok, mk, 0x7362));
    }
  };
  look_up(0);
  if (tid < kPathBits / 32) path_bits[tid] = 0u;
  __syncthreads();
  if (node > 0) {
    if (tid == 0) {
      int n = 0;
      for (int k = node; k > 0;) {
        const int p = par[k], t = tok[k];
        if (t < 0 || t >= a.V) {
          found |= kBadToken;
        } else {
          path[n++] = t;
          path_bits[t % kPathBits >> 5] |= 1u << (t & 31);
        }
        if (p < 0 || p >= k) {
          found |= kBadTree;
          break;
        }
        k = p;
      }
      n_path_s = n;
    }
    __syncthreads();
  }
  const int n_path = node > 0 ? n_path_s : 0;
  // how often a token is on the path (few pass the first test that are not: with 32 bits
  // for it in place of 4096, some lane of nearly every warp did)
  auto times = [&](int x) {
    uint32_t n = 0;
    if (path_bits[x % kPathBits >> 5] >> (x & 31) & 1u)
      for (int i = 0; i < n_path; ++i) n += path[i] == x;
    return n;
  };

  // whether a token's count and bias are the context's: those of others may hold anything
  auto marked = [&](int x) { return marks && (marks[x >> 5] >> (x & 31) & 1u); };

  const float2 ch = make_float2(a.c_hi, a.c_hi), cl = make_float2(a.c_lo, a.c_lo);
  const float far = 1048576.f / a.c_hi;
  float m_run = TV_NEG_INF, s_run = 0.f;
  for (int seg = 0; seg < blocks; seg += kSegment / 8) {
    if (seg > 0) {
      __syncthreads();                   // (the bits before are done with)
      look_up(seg);
      __syncthreads();
    }
    const int seg_end = min(blocks, seg + kSegment / 8);
    if (n_path > 0) {
      for (int k = tid; k < n_path; k += kThreads) {
        const long long p = (long long)path[k] + off - p_lo - 8ll * seg;
        if (p >= 0 && p < 8 * (seg_end - seg) && (bits[p >> 3] >> (p & 7) & 1u))
          atomicOr(reinterpret_cast<uint32_t*>(bits) + (p >> 4),
                   1u << ((p & 7) + 8 + 16 * (int)(p >> 3 & 1)));
      }
      __syncthreads();
    }
    // The bits of a step's tokens of this thread (8 a block), those that are allowed and
    // those that are marked as well.  The marked ones of a warp are shared out among its
    // threads, whichever hold them: a list of (thread, bit) codes, of which thread i has
    // the i-th, the (32 + i)-th and so on.  The first one's count and bias are asked for
    // with the logits, a step ahead of their use.
    auto token = [&](int b0, int code) {           // (code: owner lane << 5 | bit)
      return x0 + 8 * ((code >> 5) - lane) + 8 * (b0 + ((code >> 3) & 3) * kThreads) + (code & 7);
    };
    uint32_t next_ok = 0, next_mk = 0, next_count = 0;
    int next_total = 0, next_code = 0;
    float next_bias = 0.f;
    uint16_t* const list = lists + wid * 2 * kListed;
    auto ask = [&](int b0) {
      next_total = 0;
      if (b0 >= seg_end) return;
      next_ok = next_mk = 0;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const uint32_t both = bits[b0 - seg + tid + j * kThreads];
        next_ok |= (both & 0xffu) << (8 * j);
        next_mk |= (both >> 8) << (8 * j);
      }
      if (!__any_sync(0xffffffffu, next_mk != 0)) return;
      int upto = __popc(next_mk);
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      next_total = __shfl_sync(0xffffffffu, upto, 31);
      if (next_total > kListed) return;            // (each thread takes its own)
      uint16_t* const to = list + (b0 / kBlocks & 1) * kListed;
      int at = upto - __popc(next_mk);
      for (uint32_t m = next_mk; m; m &= m - 1)
        to[at++] = (uint16_t)(lane << 5 | (__ffs(m) - 1));
      __syncwarp();
      if (lane < next_total) {
        next_code = to[lane];
        if (r.counts) {
          next_count = r.counts[token(b0, next_code)];
          next_bias = r.bias[token(b0, next_code)];
        }
      }
    };
    // the element of a code, in the owner's place in shared memory
    auto element = [&](int code) {
      const int j = code >> 3 & 3, k = code & 7;
      return reinterpret_cast<E*>(stage + (j * (W / 4) + k * (int)sizeof(E) / 16) * kThreads +
                                  wid * 32 + (code >> 5)) +
             k % (16 / (int)sizeof(E));
    };
    ask(seg);
    for (int b0 = seg; b0 < seg_end; b0 += kBlocks) {
      uint32_t w[NB][W], mk = next_mk, count = next_count;
      const uint32_t ok = next_ok;
      const int total = next_total;
      int code = next_code;
      float bias = next_bias;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int k = 0; k < W; ++k) w[j][k] = next[j][k];
      fetch(b0 + kBlocks);
      ask(b0 + kBlocks);
      if (total > 0) {  // marked tokens, through shared memory
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int k = 0; k < W; k += 4)
            stage[(j * (W / 4) + k / 4) * kThreads + tid] =
                make_uint4(w[j][k], w[j][k + 1], w[j][k + 2], w[j][k + 3]);
        __syncwarp();
        const bool shared_out = total <= kListed;
        const uint16_t* const from = list + (b0 / kBlocks & 1) * kListed;
        bool asked = shared_out;
        for (int i = lane; shared_out ? i < total : mk != 0; i += 32) {
          if (!asked) {
            code = shared_out ? from[i] : lane << 5 | (__ffs(mk) - 1);
            if (r.counts) {
              count = r.counts[token(b0, code)];
              bias = r.bias[token(b0, code)];
            }
          }
          asked = false;
          mk &= mk - 1;
          E* const e = element(code);
          const int x = token(b0, code);
          const uint32_t on_path = times(x);
          if (on_path && !marked(x)) {       // (here for the path alone)
            count = 0;
            bias = 0.f;
          }
          put(e, penalised(get(e), count, bias, on_path, r));
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int k = 0; k < W; k += 4) {
            const uint4 u = stage[(j * (W / 4) + k / 4) * kThreads + tid];
            w[j][k] = u.x; w[j][k + 1] = u.y; w[j][k + 2] = u.z; w[j][k + 3] = u.w;
          }
        __syncwarp();
      }
      if (ok != (NB == 4 ? 0xffffffffu : 0xffffu)) {
#pragma unroll
        for (int j = 0; j < NB; ++j) mask_block(w[j], ok >> (8 * j) & 0xffu);
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int blk = b0 + tid + j * kThreads;
        if (blk >= lo && blk < hi) {
#pragma unroll
          for (int k = 0; k < W; k += 4)
            st16(reinterpret_cast<char*>(out + 8 * b0) + j * kThreads * 8 * (int)sizeof(E) +
                     4 * k,
                 &w[j][k]);
        }
      }
      add_blocks<L>(w, ch, cl, far, m_run, s_run);
    }
  }
  s_run = settled(s_run, m_run, ch.x, cl.x, far);
  // the blocks at the row's ends, an element a thread (one block, where the row starts and
  // ends in the same)
  if ((lo && tid < 8) || (p_hi == positions && p_lo < p_hi && hi >= lo && tid >= 8 && tid < 16)) {
    const int p = (tid < 8 ? tid : 8 * hi + (tid - 8)) - 8 * tid;   // from this thread's first
    const int x = x0 + p;
    if (x >= 0 && x < a.V) {
      uint32_t n = 0;
      float bias = 0.f;
      const bool known = marked(x);
      if (known) {
        n = r.counts[x];
        bias = r.bias[x];
      }
      const uint32_t on_path = times(x);
      float v = get(in + p);
      if (known || on_path) v = penalised(v, n, bias, on_path, r);
      if (grammar && !(grammar[x >> 5] >> (x & 31) & 1u)) v = TV_NEG_INF;
      E e;
      put(&e, v);
      out[p] = e;
      add_one(L(), get(&e), ch, cl, m_run, s_run);
    }
  }

  // the threads' (max, sum), then the cluster's CTAs' in their order
  const float wm = warp_max(m_run);
  if (lane == 0) red[0][wid] = wm;
  __syncthreads();
  float m = red[0][0];
#pragma unroll
  for (int k = 1; k < kThreads / 32; ++k) m = fmaxf(m, red[0][k]);
  float s = m_run == TV_NEG_INF ? 0.f : s_run * rescale(L(), m_run, m, ch, cl);
  s = warp_sum(s);
  if (lane == 0) red[1][wid] = s;
  if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    s = 0.f;
    for (int k = 0; k < kThreads / 32; ++k) s += red[1][k];
    if (C == 1) a.row_stats[row] = make_float2(m, s);
    else {
      const uint32_t to = map_shared(&joined[rank], 0);
      st_cluster_f32(to, m);
      st_cluster_f32(to + 4, s);
    }
    if (found) atomicOr(a.status, found);
  }
  if (C > 1) {
    cluster_sync_all();
    if (rank == 0 && tid == 0) {
      m = TV_NEG_INF;
      for (uint32_t k = 0; k < C; ++k) m = fmaxf(m, joined[k].x);
      s = 0.f;
      for (uint32_t k = 0; k < C; ++k)
        if (joined[k].x != TV_NEG_INF) s += joined[k].y * rescale(L(), joined[k].x, m, ch, cl);
      a.row_stats[row] = make_float2(m, s);
    }
  }
}

// ---- a context's arrays ----

__global__ void clear_kernel(ContextArgs c, const int32_t* __restrict__ slots, int V,
                             uint32_t* status) {
  const int s = slots[blockIdx.y], words = (V + 31) / 32;
  if (s < 0 || s >= c.n_slots) {
    if (threadIdx.x == 0) atomicOr(status, kBadSlot);
    return;
  }
  const int step = gridDim.x * blockDim.x;
  for (int x = blockIdx.x * blockDim.x + threadIdx.x; x < V; x += step) {
    c.counts[(size_t)s * V + x] = 0;
    c.bias[(size_t)s * V + x] = 0.f;
    if (x < words) c.marks[(size_t)s * words + x] = 0;
  }
}

__device__ __forceinline__ void mark(const ContextArgs& c, int s, int V, int x) {
  atomicOr(c.marks + (size_t)s * ((V + 31) / 32) + x / 32, 1u << (x & 31));
}

// Tokens [B][n] of B requests; negative ones are skipped.
__global__ void add_kernel(ContextArgs c, int kind, int B, int n,
                           const int32_t* __restrict__ slots, const int32_t* __restrict__ tokens,
                           const float* __restrict__ values, int V, uint32_t* status) {
  const long long at = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= (long long)B * n) return;
  const int b = (int)(at / n), s = slots ? slots[b] : b, x = tokens[at];
  if (s < 0 || s >= c.n_slots) {
    atomicOr(status, kBadSlot);
    return;
  }
  if (x < 0) return;
  if (x >= V) {
    atomicOr(status, kBadToken);
    return;
  }
  uint32_t* count = c.counts + (size_t)s * V + x;
  if (kind == 0) atomicOr(count, 1u);
  else if (kind == 1) atomicAdd(count, 2u);
  else c.bias[(size_t)s * V + x] = values[at];
  mark(c, s, V, x);
}

// The accepted path's tokens and the bonus token of B requests, as generated ones.
__global__ void accept_kernel(ContextArgs c, int B, int N, const int32_t* __restrict__ slots,
                              const int32_t* __restrict__ tokens,
                              const int32_t* __restrict__ path,
                              const int32_t* __restrict__ bonus, int V, uint32_t* status) {
  const long long at = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= (long long)B * (N + 1)) return;
  const int b = (int)(at / (N + 1)), k = (int)(at - (long long)b * (N + 1));
  const int s = slots ? slots[b] : b;
  if (s < 0 || s >= c.n_slots) {
    atomicOr(status, kBadSlot);
    return;
  }
  int x;
  if (k < N) {
    const int node = path[(size_t)b * N + k];
    if (node < 1 || node > N) return;      // (-1: past the accepted chain)
    x = tokens[(size_t)b * (N + 1) + node];
  } else {
    x = bonus[b];
    if (x < 0) return;                     // an invalid tree
  }
  if (x < 0 || x >= V) {
    atomicOr(status, kBadToken);
    return;
  }
  atomicAdd(c.counts + (size_t)s * V + x, 2u);
  mark(c, s, V, x);
}

}  // namespace logits
}  // namespace tvk

namespace {

template <typename L, int kThreads>
cudaError_t launch_process(const ProcessArgs& a, int C, cudaStream_t stream) {
  using namespace tvk::logits;
  const size_t smem =
      4 * ((size_t)Block<L>::kBlocks * Block<L>::kWords * kThreads + kSegment / 16 +
           kThreads / 32 * kListed + 3 * (size_t)(a.N + 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.B * (a.N + 1) * C), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // the same limit for every launch, set once per device
  static std::atomic<uint64_t> set{0};
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(set.load() >> device & 1u)) {
    e = cudaFuncSetAttribute(process_kernel<L, kThreads>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize, 96 << 10);
    if (e != cudaSuccess) return e;
    if (device < 64) set.fetch_or(1ull << device);
  }
  return cudaLaunchKernelEx(&cfg, process_kernel<L, kThreads>, a);
}

}  // namespace

int tv_launch_process(const ProcessArgs& a, int logit_is_bf16, int sm_count,
                      cudaStream_t stream) {
  // CTAs per row: those whose rounds (four CTAs an SM) take the least time, counted in steps
  // of a CTA with two and a half more for its start and end.  At V = 128256 in bf16: 8 for one
  // row and for 61 rows, 2 for 1952 (4 rounds of whole rows, 7 of halves: 194.5 us, 196 with 1,
  // 214 with 4), 1 for 7808 (744 us, 773 with 2, 851 with 4); at 864 rows of 32003 in bf16 1 (55
  // us, 58 with 2), in fp32 2 (70, 69 with 1, 82 with 4).
  const long long rows = (long long)a.B * (a.N + 1), ctas = 4ll * sm_count;
  const long long step = 8 * 256 * (logit_is_bf16 ? 4 : 2);
  const long long steps = ((long long)a.V + step - 1) / step;
  int C = 1;
  double least = 0;
  for (int c = 1; c <= tvk::logits::kMaxCluster; c *= 2) {
    const double cost = (double)((rows * c + ctas - 1) / ctas) * ((steps + c - 1) / c + 2.5);
    if (c == 1 || cost < least) {
      least = cost;
      C = c;
    }
  }
  // Threads: 512 where there is an SM for every CTA, 128 (eight CTAs an SM in place of four)
  // for many rows of one step, whose time is their start and end (30500 rows of 1003 in bf16:
  // 233 us, 364 with 256 threads; 18300 of 4000 in fp32 219, 241; but 904 for the 744 of 7808 of
  // 128256, and 795 with 512).  The steps above are those of 256 threads.  One of 512 is twice as
  // long, so that some CTAs of a row may have none: at one row of 32000 in bf16 two of four, which
  // costs a wider cluster's launch and join (5.7 us; 4.8 with four CTAs of 256 threads).
  const int threads = rows * C <= sm_count ? 512 : C == 1 && steps == 1 ? 128 : 256;
  auto run = logit_is_bf16 ? (threads == 512   ? launch_process<tvk::Bf16Logits, 512>
                              : threads == 256 ? launch_process<tvk::Bf16Logits, 256>
                                               : launch_process<tvk::Bf16Logits, 128>)
                           : (threads == 512   ? launch_process<tvk::F32Logits, 512>
                              : threads == 256 ? launch_process<tvk::F32Logits, 256>
                                               : launch_process<tvk::F32Logits, 128>);
  const cudaError_t e = run(a, C, stream);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return -5;
  }
  return 0;
}

int tv_launch_context_clear(const ContextArgs& c, int n, const int32_t* slots, int V,
                            uint32_t* status, cudaStream_t stream) {
  for (int at = 0; at < n; at += 65535) {
    const dim3 grid((V + 2047) / 2048, std::min(n - at, 65535));
    tvk::logits::clear_kernel<<<grid, 256, 0, stream>>>(c, slots + at, V, status);
  }
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

int tv_launch_context_add(const ContextArgs& c, int kind, int B, int n, const int32_t* slots,
                          const int32_t* tokens, const float* values, int V, uint32_t* status,
                          cudaStream_t stream) {
  const long long total = (long long)B * n;
  if (total == 0) return 0;
  tvk::logits::add_kernel<<<(unsigned)((total + 255) / 256), 256, 0, stream>>>(
      c, kind, B, n, slots, tokens, values, V, status);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

int tv_launch_context_accept(const ContextArgs& c, int B, int N, const int32_t* slots,
                             const int32_t* tokens, const int32_t* path, const int32_t* bonus,
                             int V, uint32_t* status, cudaStream_t stream) {
  const long long total = (long long)B * (N + 1);
  tvk::logits::accept_kernel<<<(unsigned)((total + 255) / 256), 256, 0, stream>>>(
      c, B, N, slots, tokens, path, bonus, V, status);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}
