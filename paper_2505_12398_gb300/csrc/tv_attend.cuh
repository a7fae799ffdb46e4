// tv_attend.cuh -- what the attention kernels over the 4-bit cache share: which rows and
// tokens a request has, which of a tree's rows a row sees, the queries' scaling, and the
// output.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <atomic>

#include "../../include/tv.h"
#include "tv_cache.cuh"
#include "tv_device.cuh"
#include "tv_launch.h"
#include "tv_ptx.cuh"

namespace tvk {
namespace attend {

using namespace cache;

constexpr int kMaxTokens = 1 << 30;    // tokens of a request that are looked at

// Weights are 2^(t - m + kLift), m at most kSlack below the largest t so far: within
// 2^(kSlack + kLift) = 2^14 of fp16's 65504, and down to 2^-24 of a smallest step.
constexpr float kSlack = 8.f;
constexpr float kLift = 6.f;

constexpr int kStep = 128;             // tokens of a step

struct Request {
  int len, rows, tokens;       // cached tokens, query rows, and tokens that the last row may see
  bool overrun;                // some of them are outside the page table
};

// A request with a negative length has no rows; tokens that the page table has no room for
// are left out.
__device__ __forceinline__ Request request_of(const AttendArgs& a, int b) {
  Request q;
  const int want = a.rows ? a.rows[b] : a.R;
  q.len = a.t.lengths[b];
  q.rows = q.len < 0 ? 0 : min(max(want, 0), a.R);
  q.len = max(q.len, 0);
  const long long room = min((long long)a.t.max_pages << a.c.page_shift, (long long)kMaxTokens);
  const long long all = (long long)q.len + q.rows;
  q.overrun = all > room;
  q.tokens = (int)min(all, room);
  return q;
}

// Work is cut into items, one (request, key/value head, tile of `tile` rows) each, in that
// order, and those into steps of 128 tokens.
__device__ __forceinline__ int tiles_of(const AttendArgs& a, const Request& q, int tile) {
  return (int)(((long long)q.rows * a.group + tile - 1) / tile);
}
// Tokens that a tile's rows may see.
__device__ __forceinline__ int tokens_of(const AttendArgs& a, const Request& q, int i, int tile) {
  if (a.parents) return q.tokens;
  const long long last = ((long long)(i + 1) * tile - 1) / a.group;
  return (int)min((long long)q.tokens, q.len + min(last, (long long)q.rows - 1) + 1);
}
__device__ __forceinline__ int steps_of(int tokens) { return (tokens + kStep - 1) / kStep; }
// Steps of a request's items of one head.
__device__ __forceinline__ long long head_steps(const AttendArgs& a, const Request& q, int tile) {
  const int tiles = tiles_of(a, q, tile);
  if (a.parents || tiles <= 1) return (long long)tiles * steps_of(q.tokens);
  long long n = 0;
  for (int i = 0; i < tiles; ++i) n += steps_of(tokens_of(a, q, i, tile));
  return n;
}

// A run of an item's steps [s0, s1).
struct Piece {
  Request rq;
  int b, head, m0, s0, s1;
  int tokens, steps;           // of the whole item
  long long first;             // the item's first step among all
  __device__ __forceinline__ bool whole() const { return s0 == 0 && s1 == steps; }
};

// The share of the steps that a CTA takes: [total c / ctas, total (c + 1) / ctas).
struct Shares {
  long long total, ctas;
  __device__ __forceinline__ long long begin(long long c) const { return total * c / ctas; }
  __device__ __forceinline__ int owner(long long step) const {
    return (int)(((step + 1) * ctas - 1) / total);
  }
};

// Goes through the pieces of the steps [cur, end).
struct Walker {
  int b;
  long long in_request, cur, end;
  __device__ __forceinline__ bool next(const AttendArgs& a, int tile, Piece& p) {
    while (cur < end) {
      p.rq = request_of(a, b);
      const long long per_head = head_steps(a, p.rq, tile), n = per_head * a.c.kv_heads;
      if (in_request >= n) {
        in_request -= n;
        ++b;
        continue;
      }
      p.b = b;
      p.head = (int)(in_request / per_head);
      long long at = in_request % per_head;
      int i = 0;
      if (a.parents) {
        const int each = steps_of(p.rq.tokens);
        i = (int)(at / each);
        at %= each;
        p.tokens = p.rq.tokens;
      } else {
        for (;; ++i) {
          p.tokens = tokens_of(a, p.rq, i, tile);
          if (at < steps_of(p.tokens)) break;
          at -= steps_of(p.tokens);
        }
      }
      p.steps = steps_of(p.tokens);
      p.m0 = i * tile;
      p.s0 = (int)at;
      p.first = cur - at;
      const int count = (int)min((long long)p.steps - at, end - cur);
      p.s1 = p.s0 + count;
      cur += count;
      in_request += count;
      return true;
    }
    return false;
  }
};

struct Schedule {
  long long warp_sum[32], total, offset;
  int request;
};

// The steps of all requests, and a walker over those of CTA `cta` of at most `ctas`.  By all
// threads of the block; has a barrier of it.
__device__ __forceinline__ Shares plan(const AttendArgs& a, Schedule& sh, int tile, int cta,
                                       int ctas, float pieces_per_step, Walker& w) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = blockDim.x;
  const int per = (a.B + n - 1) / n;
  long long mine = 0;
  for (int b = tid * per; b < min(a.B, (tid + 1) * per); ++b)
    mine += head_steps(a, request_of(a, b), tile) * a.c.kv_heads;
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sh.warp_sum[warp] = upto;
  __syncthreads();
  long long before = upto - mine, total = 0;
  for (int i = 0; i < (n >> 5); ++i) {
    if (i < warp) before += sh.warp_sum[i];
    total += sh.warp_sum[i];
  }
  Shares s;
  s.total = total;
  // `pieces_per_step`: of how many pieces the joining takes as long as a step.  Of an item of S
  // steps a CTA then takes sqrt(S / pieces_per_step) at least, where steps and joining together
  // are shortest.
  const long long items =
      (long long)a.B * a.c.kv_heads * (((long long)a.R * a.group + tile - 1) / tile);
  const int least = max((int)sqrtf((float)(total / items) / pieces_per_step), 1);
  s.ctas = min((long long)ctas, (total + least - 1) / least);
  w.cur = cta < s.ctas ? s.begin(cta) : 0;
  w.end = cta < s.ctas ? s.begin(cta + 1) : 0;
  if (w.cur < w.end && w.cur >= before && w.cur < before + mine) {
    long long left = w.cur - before;
    for (int b = tid * per;; ++b) {
      const long long k = head_steps(a, request_of(a, b), tile) * a.c.kv_heads;
      if (left < k) {
        sh.request = b;
        sh.offset = left;
        break;
      }
      left -= k;
    }
  }
  __syncthreads();
  w.b = sh.request;
  w.in_request = sh.offset;
  return s;
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

// Writes 0 to the rows behind each request's last, and reports lengths, row counts and
// page tables that cannot be.  By a warp, `me` of `all`.
__device__ __forceinline__ void zero_rows(const AttendArgs& a, int D, int me, int all) {
  const int lane = threadIdx.x & 31;
  const size_t row = (size_t)a.c.kv_heads * a.group * D / 8;     // 16-byte pieces
  for (int b = all < a.B ? me : me % a.B; b < a.B; b += all) {
    // (some warps for a request, or some requests for a warp)
    const int sub = all < a.B ? 0 : me / a.B, subs = all < a.B ? 1 : (all - 1 - b) / a.B + 1;
    const Request q = request_of(a, b);
    if (sub == 0 && lane == 0) {
      const int want = a.rows ? a.rows[b] : a.R;
      uint32_t bits = 0;
      if (a.t.lengths[b] < 0 || want < 0 || want > a.R) bits |= TV_STATUS_BAD_LENGTH;
      if (q.rows > 0 && q.overrun) bits |= TV_STATUS_BAD_PAGE;
      if (bits) atomicOr(a.status, bits);
    }
    uint4* const out = reinterpret_cast<uint4*>(a.out) + (size_t)b * a.R * row;
    for (int i = q.rows + sub; i < a.R; i += subs)
      for (size_t x = lane; x < row; x += 32) out[i * row + x] = make_uint4(0, 0, 0, 0);
  }
}

// Scales a row of queries whose largest magnitude is `top` by a power of two, to [2^14, 2^15)
// (or, of subnormal ones, as near as the exponent of the least normal one brings it).
struct QueryScale {
  float up0, up1;              // two factors (one power of two may be no float32)
  int e;
  bool finite;
  __device__ __forceinline__ explicit QueryScale(float top) {
    finite = top <= 3.4028234e38f;                 // (false for NaN)
    const int biased = max(__float_as_int(top) >> 23, 1);
    e = finite && top > 0.f ? biased - (127 + 14) : 0;
    const int half = -e / 2;                       // -140 <= e <= 113
    up0 = pow2i(half);
    up1 = pow2i(-e - half);
  }
  __device__ __forceinline__ float apply(float x) const { return x * up0 * up1; }
  // what makes log2(e) times the score of a product of scaled queries and keys; NaN for a
  // row that is not finite
  __device__ __forceinline__ float factor(float scale_log2e, int key_exponent) const {
    const int n = e + key_exponent, half = n / 2;
    const float most = 3.4028234e38f;              // (0 times an infinity would be no score)
    const float f = fminf(fmaxf(scale_log2e * pow2i(half) * pow2i(n - half), -most), most);
    return finite ? f : __int_as_float(0x7fffffff);
  }
};

// Waits for a phase of a barrier, unless an earlier wait gave up; `bad` becomes 1 if this does.
__device__ __forceinline__ void wait_on(uint64_t* bar, uint32_t parity, uint32_t& bad) {
  if (!mbar_try_wait(bar, parity) && !bad) bad = mbar_wait(bar, parity) ? 0u : 1u;
}

// Lets a kernel of this device take that much shared memory, once (a call costs the host 1 us).
// `done` is the kernel's own: bit i for device i.
template <typename K>
bool allow_smem(K kernel, size_t bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  const uint64_t bit = device < 64 ? 1ull << device : 0ull;
  if (bit && (done.load(std::memory_order_relaxed) & bit)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) !=
      cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  done.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

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
