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

#include "tv_device.cuh"
#include "tv_launch.h"

namespace tvk {
namespace logits {

constexpr int kThreads = 256;
constexpr int kTile = 8192;              // tokens of a CTA
constexpr int kMaxPath = 1024;           // rows of a tree at most
constexpr uint32_t kBadTree = 1u, kBadToken = 2u, kBadSlot = 256u, kBadMask = 512u;

__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

struct Row {
  const uint32_t* counts;   // of the request's slot, or nullptr
  const float* bias;
  float rep, freq, pres;
  int n_path;
};

// The logit of a marked token.
__device__ __forceinline__ float penalised(float l, int x, const Row& r, const int* path) {
  uint32_t c = 0;
  float bias = 0.f;
  if (r.counts) {
    c = r.counts[x];
    bias = r.bias[x];
  }
  uint32_t n = c >> 1;
  for (int i = 0; i < r.n_path; ++i) n += path[i] == x;
  if (n > 0 || (c & 1u)) l = l > 0.f ? __fdiv_rn(l, r.rep) : __fmul_rn(l, r.rep);
  if (n > 0) l = __fsub_rn(__fsub_rn(l, __fmul_rn(r.freq, (float)n)), r.pres);
  return __fadd_rn(l, bias);
}

template <typename L> struct Elem;
template <> struct Elem<Bf16Logits> { using type = __nv_bfloat16; };
template <> struct Elem<F32Logits> { using type = float; };

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
    w[k] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ float rounded(__nv_bfloat16*, float v) {
  return __bfloat162float(__float2bfloat16_rn(v));
}
__device__ __forceinline__ float rounded(float*, float v) { return v; }

// CTA (chunk, row): tokens [chunk * kTile, + kTile) of a row.
template <typename L, bool VEC>
__global__ void __launch_bounds__(kThreads)
    process_kernel(ProcessArgs a) {
  using E = typename Elem<L>::type;
  __shared__ uint32_t bits[kTile / 32];
  __shared__ int path[kMaxPath];
  __shared__ int n_path_s;
  __shared__ float red[2][kThreads / 32];
  const int R = a.N + 1, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int b = blockIdx.y / R, i = blockIdx.y - b * R;
  const size_t row = blockIdx.y;
  const int lo = blockIdx.x * kTile, hi = min(a.V, lo + kTile);
  const int words = (a.V + 31) / 32;
  uint32_t found = 0;

  int slot = a.slots ? a.slots[b] : a.slot0 + b;
  if (a.counts && (slot < 0 || slot >= a.n_slots)) {
    found |= kBadSlot;
    slot = -1;
  }
  Row r;
  r.counts = a.counts && slot >= 0 ? a.counts + (size_t)slot * a.V : nullptr;
  r.bias = a.bias + (size_t)max(slot, 0) * a.V;
  r.rep = a.penalties ? a.penalties[3 * b] : 1.f;
  r.freq = a.penalties ? a.penalties[3 * b + 1] : 0.f;
  r.pres = a.penalties ? a.penalties[3 * b + 2] : 0.f;
  const uint32_t* marks = r.counts ? a.marks + (size_t)slot * words : nullptr;
  int mi = a.mask_index ? a.mask_index[row] : -1;
  if (mi < -1 || mi >= a.n_masks) {
    found |= kBadMask;
    mi = -1;
  }
  const uint32_t* allow = mi >= 0 ? a.masks + (size_t)mi * words : nullptr;

  for (int w = tid; w < kTile / 32; w += kThreads)
    bits[w] = marks && lo / 32 + w < words ? marks[lo / 32 + w] : 0u;
  if (tid == 0) {       // the drafted path to this row
    int n = 0;
    const int32_t* par = a.parents + (size_t)b * R;
    for (int k = i; k > 0;) {
      const int p = par[k], t = a.tokens[(size_t)b * R + k];
      if (t < 0 || t >= a.V) found |= kBadToken;
      else path[n++] = t;
      if (p < 0 || p >= k) {
        found |= kBadTree;
        break;
      }
      k = p;
    }
    n_path_s = n;
  }
  __syncthreads();
  r.n_path = n_path_s;
  for (int k = tid; k < r.n_path; k += kThreads)
    if (path[k] >= lo && path[k] < hi) atomicOr(&bits[(path[k] - lo) / 32], 1u << (path[k] & 31));
  __syncthreads();

  const E* in = static_cast<const E*>(a.logits) + row * a.V;
  E* out = static_cast<E*>(a.out) + row * a.V;
  const float2 ch = make_float2(a.c_hi, a.c_hi), cl = make_float2(a.c_lo, a.c_lo);
  float m_run = TV_NEG_INF, s_run = 0.f;
  for (int x0 = lo + tid * 8; x0 < hi; x0 += kThreads * 8) {
    float v[8];
    load_logits<L, VEC>(reinterpret_cast<const typename L::elem*>(in), x0, a.V, v);
    const uint32_t mk = (bits[(x0 - lo) / 32] >> (x0 & 31)) & 0xffu;
    const uint32_t ok = allow ? (allow[x0 / 32] >> (x0 & 31)) & 0xffu : 0xffu;
    if (mk) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if ((mk >> k & 1u) && (VEC || x0 + k < a.V)) v[k] = penalised(v[k], x0 + k, r, path);
    }
    float m = TV_NEG_INF;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (!(ok >> k & 1u)) v[k] = TV_NEG_INF;
      v[k] = rounded(out, v[k]);
    }
    if (VEC) {
      store8(out + x0, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (x0 + k < a.V) put(out + x0 + k, v[k]);
        else v[k] = TV_NEG_INF;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, v[k]);
    if (m > m_run) {
      if (m_run != TV_NEG_INF) s_run *= L::exp_rel(m_run, m, ch.x, cl.x);
      m_run = m;
    }
    if (m_run != TV_NEG_INF) {
      float t[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = L::exp_rel(v[k], m_run, ch.x, cl.x);
      s_run += sum8(t);
    }
  }
  const float wm = warp_max(m_run);
  if (lane == 0) red[0][wid] = wm;
  __syncthreads();
  float m = red[0][0];
#pragma unroll
  for (int k = 1; k < kThreads / 32; ++k) m = fmaxf(m, red[0][k]);
  float s = m_run == TV_NEG_INF ? 0.f : s_run * L::exp_rel(m_run, m, ch.x, cl.x);
  s = warp_sum(s);
  if (lane == 0) red[1][wid] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.f;
    for (int k = 0; k < kThreads / 32; ++k) s += red[1][k];
    a.part[row * gridDim.x + blockIdx.x] = make_float2(m, s);
    if (found) atomicOr(a.status, found);
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

size_t tv_process_scratch(size_t rows, int V) {
  return rows * ((V + tvk::logits::kTile - 1) / tvk::logits::kTile);
}

int tv_launch_process(const ProcessArgs& a, int logit_is_bf16, cudaStream_t stream) {
  using namespace tvk;
  using namespace tvk::logits;
  const int rows = a.B * (a.N + 1), chunks = (a.V + kTile - 1) / kTile;
  // (a grid has at most 65535 rows of blocks)
  for (int r0 = 0; r0 < rows;) {
    const int trees = std::max(1, std::min(a.B - r0 / (a.N + 1), 65535 / (a.N + 1)));
    ProcessArgs p = a;
    const int b0 = r0 / (a.N + 1);
    const size_t off = (size_t)r0 * a.V * (logit_is_bf16 ? 2 : 4);
    p.B = trees;
    p.slots = a.slots ? a.slots + b0 : nullptr;
    p.slot0 = a.slot0 + b0;
    p.parents = a.parents + r0;
    p.tokens = a.tokens + r0;
    p.penalties = a.penalties ? a.penalties + 3 * (size_t)b0 : nullptr;
    p.mask_index = a.mask_index ? a.mask_index + r0 : nullptr;
    p.logits = static_cast<const char*>(a.logits) + off;
    p.out = static_cast<char*>(a.out) + off;
    p.part = a.part + (size_t)r0 * chunks;
    const dim3 grid(chunks, trees * (a.N + 1));
    const bool vec = a.V % 8 == 0;
    if (logit_is_bf16) {
      if (vec) process_kernel<Bf16Logits, true><<<grid, kThreads, 0, stream>>>(p);
      else process_kernel<Bf16Logits, false><<<grid, kThreads, 0, stream>>>(p);
    } else {
      if (vec) process_kernel<F32Logits, true><<<grid, kThreads, 0, stream>>>(p);
      else process_kernel<F32Logits, false><<<grid, kThreads, 0, stream>>>(p);
    }
    if (cudaGetLastError() != cudaSuccess) return -5;
    r0 += trees * (a.N + 1);
  }
  return tv_launch_merge(a.part, chunks, rows, a.c_hi, a.c_lo, a.row_stats, stream);
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
