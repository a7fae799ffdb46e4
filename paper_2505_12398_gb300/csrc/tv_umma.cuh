// tv_umma.cuh -- what the tensor-core kernels share: shared-memory and TMA
// descriptors, tcgen05 commit, allocation and tensor-memory reads, and the
// order of tiles; and the bf16 head's rounding, store and running normaliser
// (the 8-bit head, whose rows may have any length, has its own).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

#include "tv_device.cuh"
#include "tv_ptx.cuh"

namespace tvk {
namespace gemm {

constexpr int kBM = 128;          // rows of a tile per CTA (TMEM lanes)
constexpr int kBN = 256;          // columns of a tile at most (TMEM columns)
constexpr int kAccBufs = 2;                     // accumulators in tensor memory
constexpr uint32_t kTmemCols = kAccBufs * kBN;  // fp32: one column per output column

// Shared-memory matrix descriptor of a K-major operand tile written by TMA
// with the 128-byte swizzle: start address >> 4 (bits 0-13), leading byte
// offset (unused with this swizzle, set to 1; bits 16-29), stride byte offset
// 1024 B >> 4 between groups of 8 rows (bits 32-45), descriptor version 1
// (bit 46), swizzle mode 2 = 128 B (bits 61-63).  Tiles are 1024-byte aligned
// (base offset 0).  Stepping K by 16 bf16 inside the swizzled 128-byte row
// advances the start address by 32 bytes.
__device__ __forceinline__ uint64_t smem_desc(const void* p) {
  const uint64_t addr = smem_u32(p);
  return ((addr >> 4) & 0x3FFFull) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}

// 2-D tiled TMA load of box {x .. x+box0, y .. y+box1} (x in elements, a
// multiple of 64 here, so 16-byte aligned) into this CTA's shared memory,
// counted on the barrier at cluster address `bar` (kPair: the pair leader's).
template <bool kPair>
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y,
                                            uint32_t bar) {
  if constexpr (kPair)
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::"
        "bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// Row and column tile of the t-th tile in the kernel's order.
__device__ __forceinline__ void tile_coords(int t, int m_tiles, int n_tiles, int group,
                                            int& mt, int& nt) {
  const int g = group > 0 && group < m_tiles ? group : m_tiles;
  const int full = (m_tiles / g) * g * n_tiles;       // tiles in whole groups
  if (t < full) {
    const int grp = t / (g * n_tiles), r = t - grp * g * n_tiles;
    mt = grp * g + r % g;
    nt = r / g;
  } else {
    const int gt = m_tiles - (m_tiles / g) * g, r = t - full;
    mt = (m_tiles / g) * g + r % gt;
    nt = r / gt;
  }
}

// True in one lane of a converged warp.  The loops around the tensor-core and TMA
// instructions run in the whole warp with those instructions alone in the chosen
// lane: their operands (descriptors, addresses, coordinates) then stay in the
// warp's uniform registers, which the instructions read, instead of being moved
// there one by one from a divergent lane's.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(p));
  return p != 0;
}

// Arrives on `bar` (kPair: on the barrier at that offset in both CTAs) once
// every tcgen05.mma issued so far by this thread is done.
template <bool kPair>
__device__ __forceinline__ void umma_commit(uint64_t* bar) {
  if constexpr (kPair)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;" ::"r"(smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
  else
    asm volatile(
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
            smem_u32(bar))
        : "memory");
}

template <bool kPair>
__device__ __forceinline__ void tmem_alloc(uint32_t* slot) {   // a whole warp (of each CTA)
  if constexpr (kPair) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(slot)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(slot)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}

template <bool kPair>
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr) {   // the allocating warp(s)
  if constexpr (kPair)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr),
                 "r"(kTmemCols)
                 : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr),
                 "r"(kTmemCols)
                 : "memory");
}

__device__ __forceinline__ void tc_fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// 32 consecutive fp32 accumulator columns of this warp's 32 TMEM lanes (lane
// i of the warp reads TMEM lane base + i): one row per thread.  The registers
// hold the columns after tmem_wait only, which takes them through an asm
// statement of its own so that no use of them precedes it.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
        "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]),
        "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]),
        "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]),
        "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
      :
      : "memory");
}

__device__ __forceinline__ void st_global_32b(void* p, const uint32_t* w) {   // 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]),
               "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity) ? 1 : 0) != 0;
}

// Rounds 32 accumulator columns of a row to bf16, stores the first n (a
// multiple of 8) at dst (32-byte stores where `wide`: a 16-byte store writes
// half a sector) and adds the stored values to the row's running (max, sum).
__device__ __forceinline__ void store_and_sum(const uint32_t (&r)[32], __nv_bfloat16* dst, int n,
                                              bool wide, float2 ch, float2 cl, float& m_run,
                                              float& s_run) {
  uint32_t packed[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const __nv_bfloat162 h =
        __floats2bfloat162_rn(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
    packed[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  if (wide && n >= 32) {
    st_global_32b(dst, packed);
    st_global_32b(dst + 16, packed + 8);
  } else {
    uint4* d4 = reinterpret_cast<uint4*>(dst);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * i < n)
        d4[i] = make_uint4(packed[4 * i], packed[4 * i + 1], packed[4 * i + 2],
                           packed[4 * i + 3]);
  }
  // the maximum (exact on bf16 pairs) and the sum, two columns at a time;
  // columns past the end count as -inf and weigh nothing
  if (n < 32) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (2 * i >= n) packed[i] = 0xff80ff80u;   // two bf16 -inf
  }
  __nv_bfloat162 hm = *reinterpret_cast<const __nv_bfloat162*>(&packed[0]);
#pragma unroll
  for (int i = 1; i < 16; ++i)
    hm = __hmax2(hm, *reinterpret_cast<const __nv_bfloat162*>(&packed[i]));
  const float cm = fmaxf(__low2float(hm), __high2float(hm));
  if (cm > m_run) {
    if (m_run != TV_NEG_INF) s_run *= exp2_split(m_run - cm, 0.f, ch.x, cl.x);
    m_run = cm;
  }
  const float2 mm = make_float2(-m_run, -m_run);
  float2 acc[4];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float2 d = __fadd2_rn(make_float2(bf16_lo(packed[i]), bf16_hi(packed[i])), mm);
    d.x = fmaxf(d.x, -1.0e4f);      // -inf / NaN -> weight ~0
    d.y = fmaxf(d.y, -1.0e4f);
    float2 e = exp2_corrected_x2(d, ch, cl);
    if (2 * i >= n) e = make_float2(0.f, 0.f);   // (n is even)
    acc[i & 3] = i < 4 ? e : __fadd2_rn(acc[i & 3], e);
  }
  const float2 s2 = __fadd2_rn(__fadd2_rn(acc[0], acc[1]), __fadd2_rn(acc[2], acc[3]));
  s_run += s2.x + s2.y;
}


// ---- host side ----

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                 const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, fetched once through the runtime (no link
// dependency on the driver library).
inline EncodeTiled encoder() {
  static std::once_flag once;
  static EncodeTiled fn = nullptr;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiled>(p);
    else
      cudaGetLastError();
  });
  return fn;
}

}  // namespace gemm
}  // namespace tvk
