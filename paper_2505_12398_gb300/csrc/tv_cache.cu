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
// In bf16 input that distance is at least 2^-9 of the value, 2^-11 for the least middle, 1/4, so
// that y times the rounded 1 / s, rounded to multiples of 2^-12 (which puts the quotients that are
// m back on it), serves in place of the division.
//
// Bound by the bytes of the rows that are not quantised.  A warp takes 8 consecutive
// positions, aligned to 8 so that they lie in one page, 4 lanes for each: a lane loads 16
// columns, the four whole lines of a row, or stores 32 bytes, the four a line; the codes of a
// chunk's 8 positions are 128 consecutive bytes.  (With a chunk of 32 columns for each lane the
// stores of fp32 rows went to 32 lines at once, and the kernel was bound by L1: 226 us for 178
// at 32 requests of up to 4096 rows of 8 heads of 128 columns.)  With the zeros behind the shorter
// requests that is 6.7 TB/s, 0.98 of what a copy reaches; in bf16 100 us, 0.96.  16 x 2048 rows of
// bf16 are written in 34 us and read in 31, 5.0 and 5.5 TB/s (0.74 and 0.81), and of fp32 in 58
// and 52 (0.78 and 0.88): calls so short are mostly waits of loads and instructions, at 0.6 to 0.8
// of the issue slots.
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

// 16 consecutive elements, 16-byte aligned, as they come.
template <typename T>
struct Row16 {
  uint4 v[sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) v[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  }
  // as float32
  __device__ __forceinline__ void widen(float (&x)[16]) const {
    const uint32_t* const w = reinterpret_cast<const uint32_t*>(v);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (sizeof(T) == 2)
        x[i] = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
      else
        x[i] = __uint_as_float(w[i]);
    }
  }
  // the largest magnitude, NaN if one is
  __device__ __forceinline__ float top() const {
    const uint32_t* const w = reinterpret_cast<const uint32_t*>(v);
    if constexpr (sizeof(T) == 2) {
      uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
      for (int i = 1; i < 8; ++i)
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
      return max_nan(bf16_lo(m), bf16_hi(m));
    } else {
      float m = fabsf(__uint_as_float(w[0]));
#pragma unroll
      for (int i = 1; i < 16; ++i) m = max_nan(m, fabsf(__uint_as_float(w[i])));
      return m;
    }
  }
};
// Stores 32 bytes (a 16-byte store writes half a sector), or twice 16.
__device__ __forceinline__ void store_words(void* p, const uint32_t (&w)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]),
                 "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

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
// The quotients x / unit that e2m1 rounds (see above), unit = s G, 0 where the scale is 0.
__device__ __forceinline__ void quotients(float (&x)[16], float unit, __nv_bfloat16) {
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(unit));
  if (unit == 0.f) inv = 0.f;
  const float2 ii = make_float2(inv, inv), up = make_float2(2560.f, 2560.f);
#pragma unroll
  for (int j = 0; j < 16; j += 2) {        // float32 has 12 bits behind the point at 2560
    const float2 y = __fadd2_rn(__ffma2_rn(make_float2(x[j], x[j + 1]), ii, up),
                                make_float2(-2560.f, -2560.f));
    x[j] = y.x;
    x[j + 1] = y.y;
  }
}
__device__ __forceinline__ void quotients(float (&x)[16], float unit, float) {
  if (unit == 0.f) unit = __int_as_float(0x7f800000);
#pragma unroll
  for (int j = 0; j < 16; ++j) x[j] = __fdiv_rn(x[j], unit);
}

// Which request, span of positions and first of kPer strips a warp works on: a strip is kCols
// columns for each of a row's 4 lanes.  A request has whole blocks, so that one division by their
// number is all that its index takes.
template <int kCols, int kPer>
struct Part {
  int b, span, strip, strips;
  __device__ __forceinline__ Part(const CacheArgs& c, int spans, int blocks) {
    strips = 2 * c.kv_heads * c.head_dim / (4 * kCols);
    const int groups = (strips + kPer - 1) / kPer;
    b = (int)(blockIdx.x / (unsigned)blocks);
    const int i = (int)(blockIdx.x - (unsigned)b * blocks) * kWarps + (int)(threadIdx.x >> 5);
    span = i / groups;
    strip = (i - span * groups) * kPer;
    if (span >= spans) span = -1;
  }
};
// Where a column of the 2 * kv_heads * head_dim of a row (keys first) is: in the keys or values
// of the row, and in a page, in bytes from its first to the codes and the scale of its 16.
struct Where {
  int side, head;
  uint32_t x, code, scale;
  __device__ __forceinline__ Where(const CacheArgs& c, int column, int slot) {
    const uint32_t d = (uint32_t)c.head_dim, width = (uint32_t)c.kv_heads * d;
    const uint32_t block = (uint32_t)c.page_size * d * 9 / 16;
    side = (uint32_t)column >= width;
    x = (uint32_t)column - side * width;
    head = (int)(x >> (d == 128 ? 7 : 6));
    const uint32_t col = x & (d - 1);
    const uint32_t piece = col / kChunk32 * c.page_size + slot;
    const uint32_t from = (uint32_t)(2 * head + side) * block;       // below 2^31
    code = from + piece * 16 + col % kChunk32 / 2;
    scale = from + c.page_size * d / 2 + piece * 2 + (col / kGroup & 1);
  }
};

template <typename T, int kPer>
__global__ void __launch_bounds__(32 * kWarps)
    write_kernel(CacheArgs c, PageTable t, int layer, int R, int spans, int blocks,
                 const T* __restrict__ k, const T* __restrict__ v,
                 const int32_t* __restrict__ rows, uint32_t* status) {
  const int lane = threadIdx.x & 31;
  const Part<kGroup, kPer> part(c, spans, blocks);
  if (part.span < 0) return;
  const int b = part.b;
  const int len = t.lengths[b];
  const int want = rows ? rows[b] : R, r = min(max(want, 0), R);
  if (len < 0 || want != r) {
    if (part.span == 0 && part.strip == 0 && lane == 0)
      atomicOr(status, (uint32_t)TV_STATUS_BAD_LENGTH);
    if (len < 0) return;
  }
  const int off = part.span * kSpan - (len & (kSpan - 1));  // of the span's first position
  if (off >= r || r == 0) return;                           // (off may be negative)
  const int i = off + (lane >> 2);                          // this lane's row
  const bool mine = i >= 0 && i < r;
  const int slot = (int)((unsigned)len + (unsigned)i) & (c.page_size - 1);
  const size_t row = ((size_t)b * R + i) * c.kv_heads * c.head_dim;
  const T *const krow = k + row, *const vrow = v + row;
  Row16<T> raw[kPer];
#pragma unroll
  for (int n = 0; n < kPer; ++n) {
    const Where at(c, ((part.strip + n) * 4 + (lane & 3)) * kGroup, slot);
    if (mine && part.strip + n < part.strips) raw[n].load((at.side ? vrow : krow) + at.x);
  }
  const int page = page_of(c, t, b, (int)((unsigned)len + (unsigned)off));   // (the span's)
  if (page < 0) {
    if (lane == 0) atomicOr(status, (uint32_t)TV_STATUS_BAD_PAGE);
    return;
  }
  if (!mine) return;
  uint8_t* const dst = block_of(c, layer, page, 0, 0);
#pragma unroll
  for (int n = 0; n < kPer; ++n) {
    if (part.strip + n >= part.strips) break;
    const Where at(c, ((part.strip + n) * 4 + (lane & 3)) * kGroup, slot);
    const int e = exponent_of(c, layer, at.side, at.head);
    float x[kGroup], top = raw[n].top();
    raw[n].widen(x);
    if (top != top) {                      // a NaN counts as 0
      atomicOr(status, (uint32_t)TV_STATUS_NAN);
      top = 0.f;
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        x[j] = x[j] != x[j] ? 0.f : x[j];
        top = fmaxf(top, fabsf(x[j]));
      }
    }
    uint16_t s8;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;"
        : "=h"(s8)
        : "f"(0.f), "f"(__fdiv_rn(top * pow2i(-e), 6.f)));
    quotients(x, widen(decode_scales(s8)).x * pow2i(e), T());
    *reinterpret_cast<uint2*>(dst + at.code) = make_uint2(encode8(x), encode8(x + 8));
    dst[at.scale] = (uint8_t)s8;
  }
}

template <typename T, int kPer>
__global__ void __launch_bounds__(32 * kWarps)
    read_kernel(CacheArgs c, PageTable t, int layer, int n, int spans, int blocks,
                const int32_t* __restrict__ first, T* __restrict__ k, T* __restrict__ v,
                int wide, uint32_t* status) {
  constexpr int kCols = 32 / (int)sizeof(T);
  const int lane = threadIdx.x & 31;
  const Part<kCols, kPer> part(c, spans, blocks);
  if (part.span < 0) return;
  const int b = part.b;
  const int len = t.lengths[b], from = first ? first[b] : 0;
  if ((len < 0 || from < 0) && part.span == 0 && part.strip == 0 && lane == 0)
    atomicOr(status, (uint32_t)TV_STATUS_BAD_LENGTH);
  const int start = max(from, 0);
  const int count = from < 0 || len <= start ? 0 : min(len - start, n);  // rows that are read
  const int off = part.span * kSpan - (start & (kSpan - 1));
  const int i = off + (lane >> 2);
  int page = -1;
  if (count > 0 && off < count) {                                      // (off may be negative)
    page = page_of(c, t, b, (int)((unsigned)start + (unsigned)off));
    if (page < 0 && lane == 0) atomicOr(status, (uint32_t)TV_STATUS_BAD_PAGE);
  }
  if (i < 0 || i >= n) return;
  const bool there = page >= 0 && i < count;
  const int slot = (int)((unsigned)start + (unsigned)i) & (c.page_size - 1);
  const uint8_t* const src = there ? block_of(c, layer, page, 0, 0) : nullptr;
  const size_t row = ((size_t)b * n + i) * c.kv_heads * c.head_dim;
  T *const krow = k + row, *const vrow = v + row;
  uint32_t code[kPer][kCols / 8];
  uint32_t scale[kPer];
#pragma unroll
  for (int m = 0; m < kPer; ++m) {
#pragma unroll
    for (int j = 0; j < kCols / 8; ++j) code[m][j] = 0;
    scale[m] = 0;
    if (there && part.strip + m < part.strips) {
      const Where at(c, ((part.strip + m) * 4 + (lane & 3)) * kCols, slot);
      if constexpr (kCols == 16) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(src + at.code));
        code[m][0] = u.x;
        code[m][1] = u.y;
      } else {
        code[m][0] = __ldg(reinterpret_cast<const uint32_t*>(src + at.code));
      }
      scale[m] = __ldg(src + at.scale);
    }
  }
#pragma unroll
  for (int m = 0; m < kPer; ++m) {
    if (part.strip + m >= part.strips) break;
    const Where at(c, ((part.strip + m) * 4 + (lane & 3)) * kCols, slot);
    const float up = pow2i(exponent_of(c, layer, at.side, at.head));
    const uint32_t s2 = lo_lo(decode_scales(scale[m]));
    uint32_t out[8];
#pragma unroll
    for (int j = 0; j < kCols / 8; ++j) {
      uint32_t h[4];
      decode8(code[m][j], h);
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const float2 f = widen(mul2(h[z], s2));
        if constexpr (kCols == 16) {
          const __nv_bfloat162 y = __floats2bfloat162_rn(f.x * up, f.y * up);
          out[4 * j + z] = *reinterpret_cast<const uint32_t*>(&y);
        } else {
          out[2 * z] = __float_as_uint(f.x * up);
          out[2 * z + 1] = __float_as_uint(f.y * up);
        }
      }
    }
    store_words((at.side ? vrow : krow) + at.x, out, wide != 0);
  }
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
// Blocks of a request whose warps take `per` strips of 4 * cols columns each.
long long row_blocks(const CacheArgs& c, int rows, int cols, int per) {
  const long long strips = 2ll * c.kv_heads * c.head_dim / (4 * cols);
  return (spans_of(rows) * ((strips + per - 1) / per) + kWarps - 1) / kWarps;   // below 2^45
}
// Strips of a warp: with many warps several, which share what finds their rows and have their
// loads on the way together; with few one, so that more SMs have some.  Times in us with one and
// with four, requests of 61 rows (the last of 2048), 8 heads of 128 columns:
//     requests           8          16          32          64         128    16 of 2048
//     blocks of one    288         576        1152        2304        4608        16448
//     write, bf16  2.7 3.3     3.3 3.3     4.7 4.1     7.2 6.2    12.5 9.7      41  34
//     read, bf16   2.9 3.2     3.5 3.3     5.0 4.0     7.6 5.2    12.9 8.3      44  31
//     write, fp32  3.6 5.8     4.6 5.8     6.4 7.3     9.9 12.8   16.9 22.2     58  77
//     read, fp32   3.3 3.4     4.5 4.0     7.2 5.2    12.0 7.7    22.3 12.6     77  52
// (fp32 reads have twice the blocks).  Rows of fp32 are written one strip a warp at any size: four
// take 97 registers a thread, which leaves 2 CTAs an SM, and one already fills 0.81 of the issue
// slots, mostly with divisions.
constexpr int kSeveral = 4;
constexpr long long kManyBlocks = 1024;
bool several(const CacheArgs& c, int B, int rows, int cols) {
  return B * row_blocks(c, rows, cols, 1) >= kManyBlocks;
}
long long move_blocks(const CacheArgs& c) {                 // of a request; below 2^50
  return ((long long)c.layers * c.kv_heads * 2 * (c.head_dim / kChunk32) + 127) / 128;
}
}  // namespace

bool tv_cache_rows_fit(const CacheArgs& c, int B, int R) {
  const long long most = INT_MAX / kWarps;                  // (a warp's index is an int)
  if (R > INT_MAX - 2 * kSpan) return false;                // (and a row's, of the last span too)
  const long long blocks = row_blocks(c, R, 8, 1);
  return blocks <= most && blocks <= INT_MAX / (long long)B;
}
bool tv_cache_moves_fit(const CacheArgs& c, int B) {
  return move_blocks(c) <= INT_MAX / (long long)B;
}

namespace {
template <typename T, int kPer>
void launch_write(const CacheArgs& c, const PageTable& t, int layer, int B, int R, const void* k,
                  const void* v, const int32_t* rows, uint32_t* status, cudaStream_t stream) {
  const int blocks = (int)row_blocks(c, R, kGroup, kPer);
  write_kernel<T, kPer><<<(unsigned)B * (unsigned)blocks, 32 * kWarps, 0, stream>>>(
      c, t, layer, R, spans_of(R), blocks, static_cast<const T*>(k), static_cast<const T*>(v),
      rows, status);
}
template <typename T, int kPer>
void launch_read(const CacheArgs& c, const PageTable& t, int layer, int B, int n,
                 const int32_t* first, void* k, void* v, uint32_t* status, cudaStream_t stream) {
  const int blocks = (int)row_blocks(c, n, 32 / (int)sizeof(T), kPer);
  const int wide =
      ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 31u) == 0;
  read_kernel<T, kPer><<<(unsigned)B * (unsigned)blocks, 32 * kWarps, 0, stream>>>(
      c, t, layer, n, spans_of(n), blocks, first, static_cast<T*>(k), static_cast<T*>(v), wide,
      status);
}
}  // namespace

int tv_launch_cache_write(const CacheArgs& c, const PageTable& t, int layer, int B, int R,
                          int is_bf16, const void* k, const void* v, const int32_t* rows,
                          uint32_t* status, cudaStream_t stream) {
  if (!is_bf16)
    launch_write<float, 1>(c, t, layer, B, R, k, v, rows, status, stream);
  else if (several(c, B, R, kGroup))
    launch_write<__nv_bfloat16, kSeveral>(c, t, layer, B, R, k, v, rows, status, stream);
  else
    launch_write<__nv_bfloat16, 1>(c, t, layer, B, R, k, v, rows, status, stream);
  return cudaGetLastError() == cudaSuccess ? 0 : -5;
}

int tv_launch_cache_read(const CacheArgs& c, const PageTable& t, int layer, int B, int n,
                         int is_bf16, const int32_t* first, void* k, void* v, uint32_t* status,
                         cudaStream_t stream) {
  const bool many = several(c, B, n, is_bf16 ? 16 : 8);
  if (is_bf16)
    many ? launch_read<__nv_bfloat16, kSeveral>(c, t, layer, B, n, first, k, v, status, stream)
         : launch_read<__nv_bfloat16, 1>(c, t, layer, B, n, first, k, v, status, stream);
  else
    many ? launch_read<float, kSeveral>(c, t, layer, B, n, first, k, v, status, stream)
         : launch_read<float, 1>(c, t, layer, B, n, first, k, v, status, stream);
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
