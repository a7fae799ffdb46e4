// tv_attend.cuh -- what the attention kernels over the 4-bit cache share: which rows and
// tokens a request has, which of a tree's rows a row sees, the queries' scaling, and the
// output.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/tv.h"
#include "tv_cache.cuh"
#include "tv_device.cuh"
#include "tv_launch.h"

namespace tvk {
namespace attend {

using namespace cache;

constexpr int kMaxTokens = 1 << 30;    // tokens of a request that are looked at

// Weights are 2^(t - m + kLift), m at most kSlack below the largest t so far: within
// 2^(kSlack + kLift) = 2^14 of fp16's 65504, and down to 2^-24 of a smallest step.
constexpr float kSlack = 8.f;
constexpr float kLift = 6.f;

struct Request {
  int len, rows, tokens;       // cached tokens, query rows, and tokens that the last row may see
  uint32_t overrun;            // status bits
  __device__ __forceinline__ long long steps(int step) const {
    return rows > 0 ? (tokens + step - 1) / step : 0;
  }
  __device__ __forceinline__ int tiles(int group, int rows_of_tile) const {
    return (int)(((long long)rows * group + rows_of_tile - 1) / rows_of_tile);
  }
};

// A request with a negative length has no rows; tokens that the page table has no room for
// are left out.
__device__ __forceinline__ Request request_of(const AttendArgs& a, int b) {
  Request q;
  q.overrun = 0;
  const int want = a.rows ? a.rows[b] : a.R;
  q.len = a.t.lengths[b];
  q.rows = q.len < 0 ? 0 : min(max(want, 0), a.R);
  q.len = max(q.len, 0);
  const long long room = min((long long)a.t.max_pages << a.c.page_shift, (long long)kMaxTokens);
  const long long all = (long long)q.len + q.rows;
  if (all > room) q.overrun = TV_STATUS_BAD_PAGE;
  q.tokens = (int)min(all, room);
  return q;
}

// Calls see(j) for row i of a tree, its parent and so on to the root; false where that leaves
// the tree.
template <typename F>
__device__ __forceinline__ bool walk(const int32_t* parents, int i, F see) {
  for (;;) {
    see(i);
    const int p = parents[i];
    if (i == 0) return p == -1;
    if (p < 0 || p >= i) return false;
    i = p;
  }
}

// Inclusive sums over the block's threads (256 of them); returns the sum before this thread's.
__device__ __forceinline__ long long block_scan(long long* scan, long long mine,
                                                long long* total) {
  const int tid = threadIdx.x;
  scan[tid] = mine;
  __syncthreads();
  for (int d = 1; d < (int)blockDim.x; d <<= 1) {
    const long long x = tid >= d ? scan[tid - d] : 0;
    __syncthreads();
    scan[tid] += x;
    __syncthreads();
  }
  if (tid == (int)blockDim.x - 1) *total = scan[tid];
  const long long before = scan[tid] - mine;
  __syncthreads();
  return before;
}

// Writes 0 to the rows behind each request's last, and reports lengths and row counts that
// cannot be.
__device__ __forceinline__ void zero_rows(const AttendArgs& a, int D) {
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const int rows = request_of(a, b).rows;
    const int want = a.rows ? a.rows[b] : a.R;
    if (threadIdx.x == 0 && (a.t.lengths[b] < 0 || want < 0 || want > a.R))
      atomicOr(a.status, (uint32_t)TV_STATUS_BAD_LENGTH);
    const size_t row = (size_t)a.c.kv_heads * a.group * D / 8;     // 16-byte pieces
    uint4* const out = reinterpret_cast<uint4*>(a.out) + (size_t)b * a.R * row;
    for (size_t x = rows * row + threadIdx.x; x < a.R * row; x += blockDim.x)
      out[x] = make_uint4(0, 0, 0, 0);
  }
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Scales a row of queries whose largest magnitude is `top` by a power of two, to [2^14, 2^15).
struct QueryScale {
  float up0, up1;              // two factors (one power of two may be no float32)
  int e;
  bool finite;
  __device__ __forceinline__ explicit QueryScale(float top) {
    finite = top <= 3.4028234e38f;                 // (false for NaN)
    e = finite && top > 0.f ? ilogbf(top) - 14 : 0;
    const int half = -e / 2;                       // |e| <= 163
    up0 = pow2i(half);
    up1 = pow2i(-e - half);
  }
  __device__ __forceinline__ float apply(float x) const { return x * up0 * up1; }
  // what makes log2(e) times the score of a product of scaled queries and keys; NaN for a
  // row that is not finite
  __device__ __forceinline__ float factor(float scale_log2e, int key_exponent) const {
    return finite ? ldexpf(scale_log2e, e + key_exponent) : __int_as_float(0x7fffffff);
  }
};

// Four columns of row m (of M) of a (request, head), sums y over weights that sum to `sum`.
__device__ __forceinline__ void store_out(const AttendArgs& a, int b, int head, int m, int M,
                                          int col, int D, float4 y, float sum, float up) {
  if (m >= M) return;
  const float inv = sum == 0.f ? 0.f : up / sum;   // (a row that sees nothing is 0)
  const __nv_bfloat162 lo = __floats2bfloat162_rn(y.x * inv, y.y * inv);
  const __nv_bfloat162 hi = __floats2bfloat162_rn(y.z * inv, y.w * inv);
  __nv_bfloat16* const dst =
      a.out + (((size_t)b * a.R + m / a.group) * a.c.kv_heads * a.group +
               (size_t)head * a.group + m % a.group) * D + col;
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo),
                                              *reinterpret_cast<const uint32_t*>(&hi));
}

}  // namespace attend
}  // namespace tvk
