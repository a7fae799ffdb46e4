// tv_cache.cuh -- the 4-bit key/value cache's format, shared by the kernels that write,
// read and move its rows and by the attention over it.
//
// A page holds page_size tokens of every layer; its block for one layer, head and side (0
// keys, 1 values) has page_size * d * 9 / 16 bytes:
//     codes   [d / 32][page_size][16 bytes]   element 2 j of 32 in the low half of byte j
//     scales  [d / 32][page_size][2]          e4m3, one for each 16 columns
// and a column's value is e2m1 code * e4m3 scale * 2^exponent(layer, side, head).  Rows of
// one chunk of 32 columns lie together, so that the lanes of a warp that hold consecutive
// tokens load consecutive bytes.
//
// e2m1 times e4m3 has 6 significant bits and lies between 2^-10 and 2688: it is exact in
// fp16 (and in bf16), and only the power of two is left out of it.
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tv_launch.h"

namespace tvk {
namespace cache {

constexpr int kGroup = 16;               // columns of a scale
constexpr int kChunk32 = 32;             // columns of a 16-byte piece of codes
constexpr int kMaxExponent = 64;         // |exponent| at most

__device__ __forceinline__ int exponent_of(const CacheArgs& c, int layer, int side, int head) {
  if (!c.exponents) return 0;
  const int e = c.exponents[((size_t)layer * 2 + side) * c.kv_heads + head];
  return min(max(e, -kMaxExponent), kMaxExponent);
}
__device__ __forceinline__ float pow2i(int e) {          // -126 <= e <= 127
  return __int_as_float((e + 127) << 23);
}

__device__ __forceinline__ size_t block_bytes(const CacheArgs& c) {
  return (size_t)c.page_size * c.head_dim * 9 / 16;
}
// The block of a page (inside the cache) for a layer, head and side.
__device__ __forceinline__ uint8_t* block_of(const CacheArgs& c, int layer, int page, int head,
                                             int side) {
  return c.data +
         ((((size_t)layer * c.pages + page) * c.kv_heads + head) * 2 + side) * block_bytes(c);
}
// Index of the page with position pos of request b, -1 where there is none (a position
// outside the table, a page outside the cache).
__device__ __forceinline__ int page_of(const CacheArgs& c, const PageTable& t, int b, int pos) {
  const int at = pos >> c.page_shift;
  if (pos < 0 || at >= t.max_pages) return -1;
  const int page = t.table[(size_t)b * t.max_pages + at];
  return (unsigned)page < (unsigned)c.pages ? page : -1;
}

// Eight codes (a word, lowest first) as four pairs of fp16.
__device__ __forceinline__ void decode8(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
// Two scales (e4m3, the low 16 bits) as a pair of fp16.
__device__ __forceinline__ uint32_t decode_scales(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return h;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a),
                            *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t lo_lo(uint32_t a) { return __byte_perm(a, a, 0x1010); }
__device__ __forceinline__ uint32_t hi_hi(uint32_t a) { return __byte_perm(a, a, 0x3232); }
__device__ __forceinline__ float2 widen(uint32_t h) {
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if one is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

}  // namespace cache
}  // namespace tvk
