// tv_cache.cu -- rows of the 4-bit key/value cache: quantised as they are written, read
// back, and moved after a verification (sm_103a).  The format is in tv_cache.cuh.
//
// With G = 2^exponent of the row's layer, side and head, and for each 16 columns x:
//     s = e4m3(min(max |x| / (6 G), 448)),   code = e2m1(x / (s G)),
// both to the nearest, ties to even: 6 is the largest e2m1 value and 448 the largest e4m3
// one.  Both roundings are those of the exact quotients.  Dividing by G is exact.  A float32
// quotient a / 6 or y / s rounds to the same 4- or 8-bit value as the exact one: a middle m
// between two values times the divisor has at most 7 bits, so a quotient that is not m
// itself is at least ulp(a) / divisor away from it, more than half an ulp of the quotient.
// In bf16 input that distance is at least 2^-9 of the value, so that y times the rounded 1 / s,
// rounded to 13 bits (which puts the quotients that are m back on it), serves in place
// of the division.
//
// Bound by the bytes of the rows that are not quantised.  A warp takes 8 consecutive
// positions, aligned to 8 so that they lie in one page, and 4 chunks of 32 columns: it
// loads (or stores) 256 consecutive bytes of bf16 of a row, and the codes of a chunk's 8
// positions are 128 consecutive bytes.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/tv.h"
#include "tv_cache.cuh"
#include "tv_device.cuh"
#include "tv_launch.h"

namespace tvk {
namespace cache {

constexpr int kWarps = 8;
constexpr int kSpan = 8;                 // positions of a warp

// 32 consecutive elements as float32, 16-byte aligned.
__device__ __forceinline__ void load32(const __nv_bfloat16* p, float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 u = reinterpret_cast<const uint4*>(p)[i];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[8 * i + 2 * j] = bf16_lo(w[j]);
      x[8 * i + 2 * j + 1] = bf16_hi(w[j]);
    }
  }
}
__device__ __forceinline__ void load32(const float* p, float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float4 u = reinterpret_cast<const float4*>(p)[i];
    x[4 * i] = u.x;
    x[4 * i + 1] = u.y;
    x[4 * i + 2] = u.z;
    x[4 * i + 3] = u.w;
  }
}
// Stores words in pieces of 32 bytes (a 16-byte store writes half a sector) or 16.
template <int N>
__device__ __forceinline__ void store_words(void* p, const uint32_t (&w)[N], bool wide) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(
                       static_cast<uint32_t*>(p) + i),
                   "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]),
                   "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  }
}
__device__ __forceinline__ void pack32(const float (&x)[32], uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
}
__device__ __forceinline__ void pack32(const float (&x)[32], uint32_t (&w)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(x[i]);
}
template <typename T>
struct Words;
template <>
struct Words<__nv_bfloat16> { static constexpr int n = 16; };
template <>
struct Words<float> { static constexpr int n = 32; };

// Eight values as e2m1 codes, lowest first; magnitudes past 6 become 6.
__device__ __forceinline__ uint32_t encode8(const float* x) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return w;
}
// The quotient y / s that e2m1 rounds (see above); inv = 1 / s.
__device__ __forceinline__ float quotient(float y, float, float inv, __nv_bfloat16) {
  return __uint_as_float((__float_as_uint(y * inv) + 0x400u) & 0xfffff800u);
}
__device__ __forceinline__ float quotient(float y, float s, float, float) {
  return __fdiv_rn(y, s);
}

// What one lane of a warp works on: chunk `at` of the row's 2 * kv_heads * d / 32 (keys
// first), its head and side.
struct Where {
  int side, head, chunk;
  __device__ __forceinline__ Where(const CacheArgs& c, int at) {
    const int chunks = c.head_dim / kChunk32;
    chunk = at % chunks;
    at /= chunks;
    side = at >= c.kv_heads;
    head = at - side * c.kv_heads;
  }
};

template <typename T>
__global__ void __launch_bounds__(32 * kWarps)
    write_kernel(CacheArgs c, PageTable t, int layer, int B, int R, int spans,
                 const T* __restrict__ k, const T* __restrict__ v,
                 const int32_t* __restrict__ rows, uint32_t* status) {
  const int quads = 2 * c.kv_heads * (c.head_dim / kChunk32) / 4;
  const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const int q = (int)(w % quads);
  const int span = (int)(w / quads % spans);
  const int b = (int)(w / quads / spans);
  if (b >= B) return;
  const int len = t.lengths[b];
  const int want = rows ? rows[b] : R, r = min(max(want, 0), R);
  if (len < 0 || want != r) {
    if (span == 0 && q == 0 && lane == 0) atomicOr(status, (uint32_t)TV_STATUS_BAD_LENGTH);
    if (len < 0) return;
  }
  const int off = span * kSpan - (len & (kSpan - 1));       // of the span's first position
  if (off >= r) return;
  const int i = off + (lane >> 2);                          // this lane's row
  const int page = page_of(c, t, b, (int)((unsigned)len + (unsigned)off));   // (the span's)
  if (page < 0) {
    if (lane == 0) atomicOr(status, (uint32_t)TV_STATUS_BAD_PAGE);
    return;
  }
  if (i < 0 || i >= r) return;
  const int slot = (int)((unsigned)len + (unsigned)i) & (c.page_size - 1);
  const Where at(c, 4 * q + (lane & 3));
  float x[32];
  load32((at.side ? v : k) + (((size_t)b * R + i) * c.kv_heads + at.head) * c.head_dim +
             at.chunk * kChunk32,
         x);
  const float down = pow2i(-exponent_of(c, layer, at.side, at.head));
  uint32_t code[4], scale = 0;
  bool nan = false;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      float& y = x[g * kGroup + j];
      y *= down;
      nan |= y != y;
      y = y != y ? 0.f : y;
      top = fmaxf(top, fabsf(y));
    }
    uint16_t s8;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;"
        : "=h"(s8)
        : "f"(0.f), "f"(__fdiv_rn(top, 6.f)));
    scale |= (uint32_t)s8 << (8 * g);
    const float s = widen(decode_scales(s8)).x;
    const float inv = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      float& y = x[g * kGroup + j];
      y = s > 0.f ? quotient(y, s, inv, T()) : 0.f;
    }
    code[2 * g] = encode8(x + g * kGroup);
    code[2 * g + 1] = encode8(x + g * kGroup + 8);
  }
  uint8_t* const block = block_of(c, layer, page, at.head, at.side);
  const size_t piece = (size_t)at.chunk * c.page_size + slot;
  *reinterpret_cast<uint4*>(block + piece * 16) = make_uint4(code[0], code[1], code[2], code[3]);
  *reinterpret_cast<uint16_t*>(block + (size_t)c.page_size * c.head_dim / 2 + piece * 2) =
      (uint16_t)scale;
  if (nan) atomicOr(status, (uint32_t)TV_STATUS_NAN);
}

template <typename T>
__global__ void __launch_bounds__(32 * kWarps)
    read_kernel(CacheArgs c, PageTable t, int layer, int B, int n, int spans,
                const int32_t* __restrict__ first, T* __restrict__ k, T* __restrict__ v,
                int wide, uint32_t* status) {
  const int quads = 2 * c.kv_heads * (c.head_dim / kChunk32) / 4;
  const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const int q = (int)(w % quads);
  const int span = (int)(w / quads % spans);
  const int b = (int)(w / quads / spans);
  if (b >= B) return;
  const int len = t.lengths[b], from = first ? first[b] : 0;
  if ((len < 0 || from < 0) && span == 0 && q == 0 && lane == 0)
    atomicOr(status, (uint32_t)TV_STATUS_BAD_LENGTH);
  const int start = max(from, 0);
  const int count = min(max(from < 0 ? 0 : len - start, 0), n);       // rows that are read
  const int off = span * kSpan - (start & (kSpan - 1));
  const int i = off + (lane >> 2);
  int page = -1;
  if (off < count) {
    page = page_of(c, t, b, (int)((unsigned)start + (unsigned)off));
    if (page < 0 && lane == 0) atomicOr(status, (uint32_t)TV_STATUS_BAD_PAGE);
  }
  if (i < 0 || i >= n) return;
  const Where at(c, 4 * q + (lane & 3));
  float x[32];
  if (page >= 0 && i < count) {
    const int slot = (int)((unsigned)start + (unsigned)i) & (c.page_size - 1);
    const uint8_t* const block = block_of(c, layer, page, at.head, at.side);
    const size_t piece = (size_t)at.chunk * c.page_size + slot;
    const uint4 code = *reinterpret_cast<const uint4*>(block + piece * 16);
    const uint32_t s2 = decode_scales(*reinterpret_cast<const uint16_t*>(
        block + (size_t)c.page_size * c.head_dim / 2 + piece * 2));
    const float up = pow2i(exponent_of(c, layer, at.side, at.head));
    const uint32_t words[4] = {code.x, code.y, code.z, code.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t h[4];
      decode8(words[j], h);
      const uint32_t s = j < 2 ? lo_lo(s2) : hi_hi(s2);
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const float2 f = widen(mul2(h[m], s));
        x[8 * j + 2 * m] = f.x * up;
        x[8 * j + 2 * m + 1] = f.y * up;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) x[j] = 0.f;
  }
  uint32_t out[Words<T>::n];
  pack32(x, out);
  store_words((at.side ? v : k) + (((size_t)b * n + i) * c.kv_heads + at.head) * c.head_dim +
                  at.chunk * kChunk32,
              out, wide != 0);
}

// One thread for each (layer, head, side, chunk) of a request.  Moves go down (position
// j + 1 behind the root takes node path[j] >= j + 1), so that the rows of a batch are all
// loaded before the first of it is stored, and no later batch reads what an earlier one stored:
// its sources are larger than any row stored before it.
constexpr int kMoves = 8;

__global__ void __launch_bounds__(128)
    accept_kernel(CacheArgs c, PageTable t, int N, int blocks, const int32_t* __restrict__ path,
                  const int32_t* __restrict__ tau, int32_t* __restrict__ out_lengths,
                  uint32_t* status) {
  const int b = blockIdx.x / blocks, part = blockIdx.x % blocks;
  const int len = t.lengths[b], count = tau[b];
  const int32_t* const p = path + (size_t)b * N;
  const bool first = part == 0 && threadIdx.x == 0;
  if (count < 0 || len < 0) {          // an invalid tree: nothing was accepted
    if (first) {
      out_lengths[b] = len;
      if (len < 0) atomicOr(status, (uint32_t)TV_STATUS_BAD_LENGTH);
    }
    return;
  }
  // a path has to rise inside the tree
  bool ok = count <= N;
  if (ok)
    for (int j = threadIdx.x; j < count; j += blockDim.x)
      ok = ok && p[j] <= N && p[j] > (j > 0 ? p[j - 1] : 0);
  ok = __syncthreads_and(ok);
  if (first) {
    out_lengths[b] = ok ? (int)((unsigned)len + 1u + (unsigned)count) : len;
    if (!ok) atomicOr(status, (uint32_t)TV_STATUS_BAD_PATH);
  }
  if (!ok) return;
  const int chunks = c.head_dim / kChunk32;
  const long long per = (long long)c.kv_heads * 2 * chunks;
  const long long x = (long long)part * blockDim.x + threadIdx.x;
  if (x >= per * c.layers) return;
  const int layer = (int)(x / per);
  const int at = (int)(x % per);
  const int chunk = at % chunks, side = at / chunks % 2, head = at / chunks / 2;
  const size_t half = (size_t)c.page_size * c.head_dim / 2;
  // where position pos of this chunk is; nullptr outside the cache
  auto row = [&](int pos, size_t* piece) -> uint8_t* {
    const int page = page_of(c, t, b, pos);
    if (page < 0) return nullptr;
    *piece = (size_t)chunk * c.page_size + (pos & (c.page_size - 1));
    return block_of(c, layer, page, head, side);
  };
  bool bad = false;
  for (int j0 = 0; j0 < count; j0 += kMoves) {
    uint4 code[kMoves];
    uint16_t scale[kMoves];
    uint32_t move = 0;
#pragma unroll
    for (int m = 0; m < kMoves; ++m) {
      const int j = j0 + m;
      if (j >= count || p[j] == j + 1) continue;         // (already there)
      size_t piece;
      const uint8_t* const src = row((int)((unsigned)len + (unsigned)p[j]), &piece);
      if (!src) {
        bad = true;
        continue;
      }
      move |= 1u << m;
      code[m] = *reinterpret_cast<const uint4*>(src + piece * 16);
      scale[m] = *reinterpret_cast<const uint16_t*>(src + half + piece * 2);
    }
#pragma unroll
    for (int m = 0; m < kMoves; ++m) {
      if (!(move >> m & 1)) continue;
      size_t piece;
      uint8_t* const dst = row((int)((unsigned)len + 1u + (unsigned)(j0 + m)), &piece);
      if (!dst) {
        bad = true;
        continue;
      }
      *reinterpret_cast<uint4*>(dst + piece * 16) = code[m];
      *reinterpret_cast<uint16_t*>(dst + half + piece * 2) = scale[m];
    }
  }
  if (bad) atomicOr(status, (uint32_t)TV_STATUS_BAD_PAGE);
}

}  // namespace cache
}  // namespace tvk

using namespace tvk::cache;

namespace {
// Spans of `rows` rows that may start anywhere in one.
int spans_of(int rows) { return (int)(((long long)rows + 2 * kSpan - 2) / kSpan); }
long long row_blocks(const CacheArgs& c, int B, int rows) {
  const long long quads = 2ll * c.kv_heads * (c.head_dim / kChunk32) / 4;
  const long long per_request = spans_of(rows) * quads;     // below 2^28 * 2^17
  return ((long long)B * per_request + kWarps - 1) / kWarps;
}
long long move_blocks(const CacheArgs& c) {                 // of a request; below 2^50
  return ((long long)c.layers * c.kv_heads * 2 * (c.head_dim / kChunk32) + 127) / 128;
}
}  // namespace

bool tv_cache_rows_fit(const CacheArgs& c, int B, int R) {
  const long long quads = 2ll * c.kv_heads * (c.head_dim / kChunk32) / 4;
  return quads * spans_of(R) <= INT_MAX && row_blocks(c, B, R) <= INT_MAX;
}
bool tv_cache_moves_fit(const CacheArgs& c, int B) {
  return move_blocks(c) <= INT_MAX / (long long)B;
}

int tv_launch_cache_write(const CacheArgs& c, const PageTable& t, int layer, int B, int R,
                          int is_bf16, const void* k, const void* v, const int32_t* rows,
                          uint32_t* status, cudaStream_t stream) {
  const unsigned blocks = (unsigned)row_blocks(c, B, R);
  if (is_bf16)
    write_kernel<__nv_bfloat16><<<blocks, 32 * kWarps, 0, stream>>>(
        c, t, layer, B, R, spans_of(R), static_cast<const __nv_bfloat16*>(k),
        static_cast<const __nv_bfloat16*>(v), rows, status);
  else
    write_kernel<float><<<blocks, 32 * kWarps, 0, stream>>>(
        c, t, layer, B, R, spans_of(R), static_cast<const float*>(k),
        static_cast<const float*>(v), rows, status);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

int tv_launch_cache_read(const CacheArgs& c, const PageTable& t, int layer, int B, int n,
                         int is_bf16, const int32_t* first, void* k, void* v, uint32_t* status,
                         cudaStream_t stream) {
  const unsigned blocks = (unsigned)row_blocks(c, B, n);
  const int wide =
      ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 31u) == 0;
  if (is_bf16)
    read_kernel<__nv_bfloat16><<<blocks, 32 * kWarps, 0, stream>>>(
        c, t, layer, B, n, spans_of(n), first, static_cast<__nv_bfloat16*>(k),
        static_cast<__nv_bfloat16*>(v), wide, status);
  else
    read_kernel<float><<<blocks, 32 * kWarps, 0, stream>>>(
        c, t, layer, B, n, spans_of(n), first, static_cast<float*>(k), static_cast<float*>(v),
        wide, status);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

int tv_launch_cache_accept(const CacheArgs& c, const PageTable& t, int B, int N,
                           const int32_t* path, const int32_t* tau, int32_t* out_lengths,
                           uint32_t* status, cudaStream_t stream) {
  const int blocks = (int)move_blocks(c);
  accept_kernel<<<(unsigned)B * (unsigned)blocks, 128, 0, stream>>>(c, t, N, blocks, path, tau,
                                                                    out_lengths, status);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}
