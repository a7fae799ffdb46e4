// tv_norm.cu -- the target model's final root-mean-square norm with the residual's
// addition, and the 8-bit operands of the LM head (sm_103a).
//
// Norm of a row:  h = x + r;  y = h w / sqrt(mean(h^2) + eps), with h and the sums in
// fp32 and the new residual stream h rounded once to the type of x.  y is rounded once
// to bf16, or, in groups of 128 columns, to e4m3 after a product with 1 / s, where s =
// max(max|y|, 2^-100) / 448 is the group's scale (448 is the largest e4m3 value; the floor
// keeps 1 / s finite for rows of zeros).  The inverse is rounded once for the group, so that
// a quotient next to the middle of two values may become either.  Weights take the same
// rounding with one scale for each 128 x 128 block.
//
// Both are bound by their bytes.  The norm keeps a row in the registers of one CTA (8
// consecutive columns, 16 bytes of bf16, per thread and step), so x and r are read once;
// 16 neighbouring threads hold a group, whose largest magnitude is four shuffles away.
// The quantiser keeps a block in the registers of one CTA.  Measured (GB300, bf16, e4m3
// out): norm of 7808 x 4096, 38.6 us, 5.8 TB/s (floor 33.2); of 61 x 4096, 2.3 us of the
// GPU; quantiser of 32000 x 2048, 34.9 us, 5.6 TB/s (29.0); of 128256 x 4096, 242 us, 6.5
// TB/s (232.5).  A ring of TMA copies with persistent CTAs in the norm's place took 40.8 us
// at 7808 x 4096 and 72 us for 36 at 30000 x 1024.  Rows of more than 16384 columns take eight
// steps of 1024 threads, whose 64 registers do not hold a thread's 64 values (92 to 732 bytes
// spilled): 4000 x 16384 76.6 us, 4000 x 16392 99.1, 2000 x 32768 92.8, 1000 x 65536 107 (floors
// 67.7).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "tv_device.cuh"
#include "tv_launch.h"

namespace tvk {
namespace norm {

constexpr int kGroup = 128;              // columns that share a scale
constexpr int kVec = 8;                  // columns of a thread per step
constexpr float kE4m3Max = 448.f;
constexpr float kLeast = 7.888609052210118e-31f;   // 2^-100
constexpr int kMaxSteps = 8;             // steps of a row's CTA at most

// Four values as e4m3 bytes, lowest first, to the nearest (ties to even); values past
// +-448 become +-448, NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// The larger magnitude; NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Eight consecutive elements of either type, 16-byte aligned (bf16) or 2 x 16 (fp32).
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = bf16_lo(w[k]);
    v[2 * k + 1] = bf16_hi(w[k]);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
// The same before it is widened, so that many can be on their way.
template <typename X>
struct Raw8 {
  uint4 v[sizeof(X) / 2];
  __device__ __forceinline__ void load(const X* p) {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(X) / 2); ++k) v[k] = reinterpret_cast<const uint4*>(p)[k];
  }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
    load8(reinterpret_cast<const X*>(v), f);
  }
};
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

// One CTA per row, or one warp (blockDim.x = 32) for each of blockDim.y.  Every element of the
// row is read before any is written, so out_residual may be x or residual.  kSteps *
// blockDim.x * 8 >= K.
template <typename X, typename W, bool kQuant, int kSteps>
__global__ void __launch_bounds__(kSteps < kMaxSteps ? 512 : 1024)
    rms_norm_kernel(const X* x, const X* residual, const W* __restrict__ weight, int M, int K,
                    float eps, X* out_residual, __nv_bfloat16* __restrict__ out_bf16,
                    uint8_t* __restrict__ out_e4m3, float* __restrict__ out_scales) {
  __shared__ float red[32];
  const size_t row = (size_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= (size_t)M) return;                  // (a whole warp, with no barrier ahead)
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, nw = blockDim.x >> 5;
  float h[kSteps][kVec];
  float sq = 0.f;
  // all of a thread's loads at once (of the longest rows, more than the registers hold, a
  // step's); columns past the end read the last ones
  constexpr int kAtOnce = kSteps < kMaxSteps ? kSteps : 1;
#pragma unroll
  for (int i0 = 0; i0 < kSteps; i0 += kAtOnce) {
    Raw8<X> rx[kAtOnce], rr[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int c = min(((i0 + i) * (int)blockDim.x + tid) * kVec, K - kVec);
      rx[i].load(x + row * K + c);
      if (residual) rr[i].load(residual + row * K + c);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      float (&hi)[kVec] = h[i0 + i];
      rx[i].widen(hi);
      if (residual) {
        float r[kVec];
        rr[i].widen(r);
#pragma unroll
        for (int k = 0; k < kVec; ++k) hi[k] += r[k];
      }
      float t[kVec];
#pragma unroll
      for (int k = 0; k < kVec; ++k) t[k] = hi[k] * hi[k];
      if (((i0 + i) * (int)blockDim.x + tid) * kVec < K) sq += sum8(t);
    }
  }
  sq = warp_sum(sq);
  if (nw > 1) {
    if (lane == 0) red[wid] = sq;
    __syncthreads();
    sq = warp_sum(lane < nw ? red[lane] : 0.f);    // (the same order in every warp)
  }
  const float inv = 1.f / sqrtf(sq / (float)K + eps);
  const int groups = (K + kGroup - 1) / kGroup;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int c = (i * (int)blockDim.x + tid) * kVec;
    const bool in = c < K;
    if (in && out_residual) store8(out_residual + row * K + c, h[i]);
    float w[kVec];
    if (in) load8(weight + c, w);
#pragma unroll
    for (int k = 0; k < kVec; ++k) h[i][k] = in ? h[i][k] * inv * w[k] : 0.f;
    if constexpr (!kQuant) {
      if (in) store8(out_bf16 + row * K + c, h[i]);
    } else {
      float m = 0.f;
#pragma unroll
      for (int k = 0; k < kVec; ++k) m = max_nan(m, fabsf(h[i][k]));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float s = max_nan(m, kLeast) / kE4m3Max;
      const float is = 1.f / s;
      if (in) {
        const uint32_t lo = e4m3x4(h[i][0] * is, h[i][1] * is, h[i][2] * is, h[i][3] * is);
        const uint32_t hi = e4m3x4(h[i][4] * is, h[i][5] * is, h[i][6] * is, h[i][7] * is);
        *reinterpret_cast<uint2*>(out_e4m3 + row * K + c) = make_uint2(lo, hi);
        if ((lane & 15) == 0) out_scales[row * groups + c / kGroup] = s;
      }
    }
  }
}

// One CTA per 128 x 128 block: 8 threads a row (16 columns each), 32 rows a step.
template <typename X>
__global__ void __launch_bounds__(256, sizeof(X) == 2 ? 3 : 2)
    quantize_block_kernel(const X* __restrict__ w, int V, int K, uint8_t* __restrict__ out,
                          float* __restrict__ scales) {
  __shared__ float red[8];
  const int groups = (K + kGroup - 1) / kGroup;
  const int br = blockIdx.x / groups, bc = blockIdx.x - br * groups;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int c = bc * kGroup + (tid & 7) * 16;
  float v[4][2][kVec];
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = br * kGroup + i * 32 + (tid >> 3);
    const bool in = r < V && c < K;               // (K is a multiple of 16)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (in) {
        load8(w + (size_t)r * K + c + j * kVec, v[i][j]);
      } else {
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[i][j][k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) m = max_nan(m, fabsf(v[i][j][k]));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) red[wid] = m;
  __syncthreads();
  m = red[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) m = max_nan(m, red[k]);
  const float s = max_nan(m, kLeast) / kE4m3Max, is = 1.f / s;
  if (tid == 0) scales[blockIdx.x] = s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = br * kGroup + i * 32 + (tid >> 3);
    if (r < V && c < K) {
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* p = &v[i][j >> 1][(j & 1) * 4];
        o[j] = e4m3x4(p[0] * is, p[1] * is, p[2] * is, p[3] * is);
      }
      *reinterpret_cast<uint4*>(out + (size_t)r * K + c) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

template <typename X, typename W, bool kQuant>
int launch_norm(int M, int K, const void* x, const void* residual, const void* weight, float eps,
                void* out_residual, void* out, float* out_scales, int sm_count,
                cudaStream_t stream) {
  // Few rows: a thread for every 8 columns, up to 512 (61 x 4096: 2.3 us, 2.7 with half as
  // many).  Many: four steps of a thread in bf16, two in fp32, so that its loads are on
  // their way at once and an SM holds more rows, whose waits for their sums and stores
  // overlap (15625 x 4096: 79 us with 512 threads, 70 with 256, 68 with 128, where 66 is
  // the floor).
  const int vecs = (K + kVec - 1) / kVec;
  const int aim = M <= 2 * sm_count ? 1 : sizeof(X) == 2 ? 4 : 2;
  int steps = 1;
  while (steps < kMaxSteps && ((steps < aim && vecs > 64 * steps) ||
                               (vecs + steps - 1) / steps > 512))
    steps *= 2;
  const int threads = std::min(1024, ((vecs + steps - 1) / steps + 31) / 32 * 32);
  // Rows of up to 256 columns, a warp each: eight to a CTA where there are many (65536 x 128:
  // 35 us with a CTA a row, bound by their launches; 18 with eight).
  const int together = threads == 32 && M > 2 * sm_count ? 8 : 1;
  auto run = [&](auto kernel) {
    kernel<<<(M + together - 1) / together, dim3(threads, together), 0, stream>>>(
        static_cast<const X*>(x), static_cast<const X*>(residual), static_cast<const W*>(weight),
        M, K, eps, static_cast<X*>(out_residual), kQuant ? nullptr : static_cast<__nv_bfloat16*>(out),
        kQuant ? static_cast<uint8_t*>(out) : nullptr, out_scales);
  };
  switch (steps) {
    case 1: run(rms_norm_kernel<X, W, kQuant, 1>); break;
    case 2: run(rms_norm_kernel<X, W, kQuant, 2>); break;
    case 4: run(rms_norm_kernel<X, W, kQuant, 4>); break;
    default: run(rms_norm_kernel<X, W, kQuant, 8>); break;
  }
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

template <typename X>
int launch_norm_of(int M, int K, const void* x, const void* residual, const void* weight,
                   int weight_is_bf16, float eps, void* out_residual, void* out,
                   float* out_scales, int sm_count, cudaStream_t stream) {
  auto run = weight_is_bf16
                 ? (out_scales ? launch_norm<X, __nv_bfloat16, true>
                               : launch_norm<X, __nv_bfloat16, false>)
                 : (out_scales ? launch_norm<X, float, true> : launch_norm<X, float, false>);
  return run(M, K, x, residual, weight, eps, out_residual, out, out_scales, sm_count, stream);
}

}  // namespace norm
}  // namespace tvk

int tv_norm_max_columns() { return tvk::norm::kMaxSteps * 1024 * tvk::norm::kVec; }

int tv_launch_rms_norm(int M, int K, int x_is_bf16, const void* x, const void* residual,
                       int weight_is_bf16, const void* weight, float eps, void* out_residual,
                       void* out, float* out_scales, int sm_count, cudaStream_t stream) {
  auto run =
      x_is_bf16 ? tvk::norm::launch_norm_of<__nv_bfloat16> : tvk::norm::launch_norm_of<float>;
  return run(M, K, x, residual, weight, weight_is_bf16, eps, out_residual, out, out_scales,
             sm_count, stream);
}

int tv_launch_quantize_weight(int V, int K, int is_bf16, const void* weight, void* out,
                              float* out_scales, cudaStream_t stream) {
  using namespace tvk::norm;
  const unsigned blocks =
      (unsigned)((V + kGroup - 1) / kGroup) * (unsigned)((K + kGroup - 1) / kGroup);
  if (is_bf16)
    quantize_block_kernel<<<blocks, 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(weight), V,
                                                      K, static_cast<uint8_t*>(out), out_scales);
  else
    quantize_block_kernel<<<blocks, 256, 0, stream>>>(static_cast<const float*>(weight), V, K,
                                                      static_cast<uint8_t*>(out), out_scales);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}
