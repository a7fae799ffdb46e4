// tv_gemm8.cu -- the target model's LM head on 8-bit operands with block scales
// (sm_103a).
//
//   l[i][v] = sum_g sa[i][g] sw[v / 128][g] P_g[i][v],   P_g = sum_{k in g} qa[i][k] qw[v][k]
//
// over groups g of 128 columns of K: hidden states and output embedding in e4m3,
// one fp32 scale for each (row, group) of the first and each 128 x 128 block of the
// second.  The logits are rounded once to bf16; on request each stored row's
// normaliser (max, sum of 2^((l - max) c)) comes with them.
//
// One persistent kernel, one CTA per SM (SM pairs above 128 rows), with the ring,
// tile order and roles of the bf16 LM head.  What differs: the scales are general fp32
// numbers, so the tensor cores' own block scaling (powers of two) does not serve.  A
// stage holds one group of K (128 bytes of a row, one swizzle row); its four
// tcgen05.mma of kind::f8f6f4 start from zero in one of two tensor-memory
// accumulators of up to 256 columns, and 16 warps add s P_g to fp32 sums in their
// registers (64 columns of a row per thread) while the tensor cores work on the next
// group.  Every wait is bounded, as there.
#include <limits.h>

#include <algorithm>

#include "tv_launch.h"
#include "tv_umma.cuh"

namespace tvk {
namespace gemm8 {

using namespace gemm;

constexpr int kGroup = 128;       // K per scale, and per stage: 128 bytes, one swizzle row
constexpr int kUmmaK = 32;        // K per tcgen05.mma of kind::f8f6f4
constexpr int kMaxStages = 8;
constexpr size_t kRingBytes = 200u << 10;
constexpr size_t kGroupBytes = 32u << 20;       // H bytes of a group of row tiles
constexpr int kParts = 4;                       // epilogue warps per TMEM lane quarter
constexpr int kEpiWarps = 4 * kParts;
constexpr int kThreads = 64 + 32 * kEpiWarps;   // TMA warp, MMA warp, epilogue warps
constexpr size_t kSmemBytes = kRingBytes + 1024;
constexpr int kChunks = kBN / (32 * kParts);    // 32-column chunks of a thread at most

// Instruction descriptor of tcgen05.mma kind::f8f6f4: fp32 accumulator (bits 4-5 =
// 1), e4m3 A and B (bits 7-9, 10-12 = 0), both K-major, N >> 3 in bits 17-22, M >> 4
// in bits 24-28.
__device__ __forceinline__ uint32_t instr_desc(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <bool kPair>
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc,
                                          uint32_t accumulate) {
  if constexpr (kPair)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Launch shape: tile width, H rows a TMA box takes per CTA, ring stages.
struct Shape {
  int bn, a_box, stages;
  __host__ __device__ uint32_t a_bytes() const { return (uint32_t)a_box * kGroup; }
  __host__ __device__ uint32_t b_bytes(bool pair) const {
    return (uint32_t)(pair ? bn / 2 : bn) * kGroup;
  }
};

// The widest stores that every row's 32-column chunks allow.
enum { kStore2 = 0, kStore16 = 1, kStore32 = 2 };

// Rounds 32 columns of a row to bf16 and stores the first n.
__device__ __forceinline__ void store_row(const float2 (&a)[16], __nv_bfloat16* dst, int n,
                                          int mode, uint32_t (&packed)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a[i].x, a[i].y);
    packed[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  if (mode == kStore32 && n >= 32) {
    st_global_32b(dst, packed);
    st_global_32b(dst + 16, packed + 8);
  } else if (mode != kStore2) {          // (n is a multiple of 8)
    uint4* d4 = reinterpret_cast<uint4*>(dst);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * i < n)
        d4[i] = make_uint4(packed[4 * i], packed[4 * i + 1], packed[4 * i + 2],
                           packed[4 * i + 3]);
  } else {
    uint16_t* d = reinterpret_cast<uint16_t*>(dst);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (2 * i < n) d[2 * i] = (uint16_t)packed[i];
      if (2 * i + 1 < n) d[2 * i + 1] = (uint16_t)(packed[i] >> 16);
    }
  }
}

// Adds the first n of 32 stored values to a row's running (max, sum).
__device__ __forceinline__ void sum_row(uint32_t (&packed)[16], int n, float2 ch, float2 cl,
                                        float& m_run, float& s_run) {
  if (n < 32) {       // columns past the end count as -inf
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (2 * i >= n) packed[i] = (packed[i] & 0xffff0000u) | 0xff80u;
      if (2 * i + 1 >= n) packed[i] = (packed[i] & 0xffffu) | 0xff800000u;
    }
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
  if (m_run == TV_NEG_INF) return;      // nothing finite yet
  const float2 mm = make_float2(-m_run, -m_run);
  float2 acc[4];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float2 d = __fadd2_rn(make_float2(bf16_lo(packed[i]), bf16_hi(packed[i])), mm);
    float2 e = exp2_corrected_x2(d, ch, cl);
    e.x = fmaxf(e.x, 0.f);              // (-inf and NaN weigh nothing)
    e.y = fmaxf(e.y, 0.f);
    acc[i & 3] = i < 4 ? e : __fadd2_rn(acc[i & 3], e);
  }
  const float2 s2 = __fadd2_rn(__fadd2_rn(acc[0], acc[1]), __fadd2_rn(acc[2], acc[3]));
  s_run += s2.x + s2.y;
}

// The tiles t = first, first + step, ... of the logits (in the order of tile_coords)
// and, with kStats, each row's (max, sum) over a tile's columns in part[row][tile].
// kPair: launched as clusters of two CTAs.
template <bool kPair, bool kStats>
__global__ void __launch_bounds__(kThreads, 1)
    lm_head8_kernel(const __grid_constant__ CUtensorMap map_h,
                    const __grid_constant__ CUtensorMap map_w, const float* __restrict__ h_scale,
                    const float* __restrict__ w_scale, int M, int V, int K, Shape shape,
                    float c_hi, float c_lo, __nv_bfloat16* __restrict__ logits,
                    float2* __restrict__ part, int m_tiles, int n_tiles, int group, int store,
                    uint32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kMaxStages];   // (kPair: the leader's are used)
  __shared__ __align__(8) uint64_t empty_bar[kMaxStages];
  __shared__ __align__(8) uint64_t acc_full[kAccBufs];    // a group's product is ready
  __shared__ __align__(8) uint64_t acc_empty[kAccBufs];   // it is read (kPair: the leader's)
  __shared__ __align__(8) uint64_t drain_bar;
  __shared__ __align__(8) uint64_t ms_full[4], ms_empty[4];
  __shared__ float2 part_ms[kParts - 1][kBM];
  __shared__ uint32_t tmem_slot;
  __shared__ int failed;
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = kPair ? cluster_rank() : 0u;
  const int first = kPair ? (int)blockIdx.x >> 1 : (int)blockIdx.x;
  const int step = kPair ? (int)gridDim.x >> 1 : (int)gridDim.x;
  const int tile_rows = kPair ? 2 * kBM : kBM;
  const int bn = shape.bn, bn_own = kPair ? bn / 2 : bn;
  const uint32_t n_stages = (uint32_t)shape.stages;
  const uint32_t a_bytes = shape.a_bytes(), stage_bytes = a_bytes + shape.b_bytes(kPair);
  const int nkb = (K + kGroup - 1) / kGroup;
  const int n_total = m_tiles * n_tiles;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < n_stages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int k = 0; k < kAccBufs; ++k) {
      mbar_init(&acc_full[k], 1);
      mbar_init(&acc_empty[k], kPair ? 2 * kEpiWarps : kEpiWarps);
    }
    mbar_init(&drain_bar, 1);
    for (int k = 0; k < 4; ++k) {
      mbar_init(&ms_full[k], kParts - 1);
      mbar_init(&ms_empty[k], 1);
    }
    failed = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc<kPair>(&tmem_slot);
  tc_fence_before();
  __syncthreads();
  if constexpr (kPair) cluster_sync_all();   // the peer's barriers and tensor memory are ready
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  asm volatile("griddepcontrol.launch_dependents;");

  if (warp == 0) {
    // ---- TMA producer: one ring across all of this CTA's tiles ----
    uint32_t it = 0, s = 0, ph = 0;
    bool ok = true;
    for (int t = first; t < n_total && ok; t += step) {
      int mt, nt;
      tile_coords(t, m_tiles, n_tiles, group, mt, nt);
      const int m0 = mt * tile_rows + (int)rank * kBM, n0 = nt * bn + (int)rank * bn_own;
      for (int kb = 0; kb < nkb; ++kb, ++it) {
        if (it >= n_stages && !wait_warp(&empty_bar[s], ph ^ 1u)) {
          ok = false;
          break;
        }
        uint8_t* a = smem + s * stage_bytes;
        uint32_t bar = smem_u32(&full_bar[s]);
        if constexpr (kPair) bar = map_shared(&full_bar[s], 0);
        if (elect_one()) {
          if (rank == 0) mbar_arrive_expect_tx(&full_bar[s], kPair ? 2 * stage_bytes : stage_bytes);
          tma_load_2d<kPair>(a, &map_h, kb * kGroup, m0, bar);
          tma_load_2d<kPair>(a + a_bytes, &map_w, kb * kGroup, n0, bar);
        }
        __syncwarp();
        if (++s == n_stages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) failed = 1;
    if (rank == 0)      // the copies issued last have landed before the CTA may exit
      for (uint32_t j = it > n_stages ? it - n_stages : 0u; j < it; ++j)
        if (!wait_warp(&full_bar[j % n_stages], (j / n_stages) & 1)) failed = 1;
  } else if (warp == 1) {
    // ---- tensor-core issue: each group's product into the accumulators in turn ----
    if (rank == 0) {
      const uint32_t idesc = instr_desc(tile_rows, bn);
      const uint64_t desc0 = smem_desc(smem);
      uint32_t s = 0, ph = 0, g = 0;
      bool ok = true;
      for (int t = first; t < n_total && ok; t += step) {
        for (int kb = 0; kb < nkb; ++kb, ++g) {
          const uint32_t acc = g & 1u;
          if (g >= kAccBufs) {
            const uint32_t par = ((g >> 1) - 1) & 1;
            const bool got = kPair ? mbar_wait_cluster(&acc_empty[acc], par)
                                   : mbar_wait(&acc_empty[acc], par);
            if (!__all_sync(0xffffffffu, got)) {
              ok = false;
              break;
            }
          }
          if (!wait_warp(&full_bar[s], ph)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem + acc * (uint32_t)kBN;
          const uint64_t da = desc0 + (uint64_t)((s * stage_bytes) >> 4);
          const uint64_t db = da + (uint64_t)(a_bytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kGroup / kUmmaK; ++k) {
              const uint64_t off = (uint64_t)((k * kUmmaK) >> 4);
              umma_e4m3<kPair>(d, da + off, db + off, idesc, k > 0 ? 1u : 0u);
            }
            umma_commit<kPair>(&acc_full[acc]);
            umma_commit<kPair>(&empty_bar[s]);
          }
          __syncwarp();
          if (++s == n_stages) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) failed = 1;
      // every MMA issued has finished before tensor memory is freed
      if (elect_one()) umma_commit<kPair>(&drain_bar);
      __syncwarp();
    }
    // (kPair, the peer: the leader's last signal)
    if (!wait_warp(&drain_bar, 0)) failed = 1;
  } else {
    // ---- scaled sums: one row per thread, every fourth 32-column chunk ----
    const int q = warp & 3;                       // the TMEM lane quarter of this warp
    const int mine = (warp - 2) >> 2;
    const float2 ch = make_float2(c_hi, c_hi), cl = make_float2(c_lo, c_lo);
    const int w_blocks = (V + kGroup - 1) / kGroup;
    uint32_t g = 0;
    int j = 0;
    bool ok = true;
    for (int t = first; t < n_total && ok; t += step, ++j) {
      int mt, n_tile;
      tile_coords(t, m_tiles, n_tiles, group, mt, n_tile);
      const int n0 = n_tile * bn;
      const int row0 = mt * tile_rows + (int)rank * kBM + q * 32, row = row0 + lane;
      const bool live = row0 < M;                 // (the same in the whole warp)
      const uint32_t tbase = tmem + ((uint32_t)(q * 32) << 16);
      const float* sa = h_scale + (size_t)min(row, M - 1) * nkb;
      const float* sw[kChunks];
      float2 sum[kChunks][16];
      float sa_next = __ldg(sa), sw_next[kChunks];
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        const int blk = min((n0 + 32 * (mine + kParts * k)) / kGroup, w_blocks - 1);
        sw[k] = w_scale + (size_t)blk * nkb;
        sw_next[k] = __ldg(sw[k]);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[k][i] = make_float2(0.f, 0.f);
      }
      for (int kb = 0; kb < nkb; ++kb, ++g) {
        float s[kChunks];
#pragma unroll
        for (int k = 0; k < kChunks; ++k) s[k] = sa_next * sw_next[k];
        if (kb + 1 < nkb) {                       // the next group's scales
          sa_next = __ldg(sa + kb + 1);
#pragma unroll
          for (int k = 0; k < kChunks; ++k) sw_next[k] = __ldg(sw[k] + kb + 1);
        }
        const uint32_t acc = g & 1u;
        if (!wait_warp(&acc_full[acc], (g >> 1) & 1)) {
          if (lane == 0) failed = 1;
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
          const int c = 32 * (mine + kParts * k);
          const bool last = k == kChunks - 1 || c + 32 * kParts >= bn;
          if (c < bn) {                           // (the same in the whole warp)
            uint32_t r[32];
            if (live) {
              __syncwarp();
              tmem_ld32(tbase + acc * (uint32_t)kBN + (uint32_t)c, r);
              tmem_wait(r);
            }
            if (last) {       // all read: this accumulator may be overwritten
              tc_fence_before();
              __syncwarp();
              if (lane == 0) {
                if constexpr (kPair) mbar_arrive_remote(map_shared(&acc_empty[acc], 0));
                else mbar_arrive(&acc_empty[acc]);
              }
            }
            if (live) {
              const float2 ss = make_float2(s[k], s[k]);
#pragma unroll
              for (int i = 0; i < 16; ++i)
                sum[k][i] = __ffma2_rn(
                    make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), ss,
                    sum[k][i]);
            }
          }
        }
      }
      if (!ok) break;
      float m_run = TV_NEG_INF, s_run = 0.f;
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        const int c = 32 * (mine + kParts * k), col0 = n0 + c;
        const int n = min(32, V - col0);          // columns of the chunk that exist
        if (c < bn && row < M && n > 0) {
          uint32_t packed[16];
          store_row(sum[k], logits + (size_t)row * V + col0, n, store, packed);
          if constexpr (kStats) sum_row(packed, n, ch, cl, m_run, s_run);
        }
      }
      if constexpr (kStats) {    // one partial per row and tile from the quarter's warps
        if (mine > 0) {
          if (j > 0 && !wait_warp(&ms_empty[q], (j - 1) & 1)) {
            if (lane == 0) failed = 1;
            break;
          }
          part_ms[mine - 1][q * 32 + lane] = make_float2(m_run, s_run);
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms_full[q]);
        } else {
          if (!wait_warp(&ms_full[q], j & 1)) {
            if (lane == 0) failed = 1;
            break;
          }
          float2 o[kParts - 1];
          float mx = m_run;
#pragma unroll
          for (int k = 0; k < kParts - 1; ++k) {
            o[k] = part_ms[k][q * 32 + lane];
            mx = fmaxf(mx, o[k].x);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms_empty[q]);
          float total = 0.f;
          if (m_run != TV_NEG_INF) total = s_run * exp2_split(m_run - mx, 0.f, c_hi, c_lo);
#pragma unroll
          for (int k = 0; k < kParts - 1; ++k)
            if (o[k].x != TV_NEG_INF) total += o[k].y * exp2_split(o[k].x - mx, 0.f, c_hi, c_lo);
          if (row < M) part[(size_t)row * n_tiles + n_tile] = make_float2(mx, total);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // (the leader's drain is over: no MMA or copy still touches either CTA)
  if constexpr (kPair) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<kPair>(tmem);
  }
  if (threadIdx.x == 0 && failed) atomicOr(status, 32u);
}

}  // namespace gemm8
}  // namespace tvk

// --------------------------------------------------------------- launcher --

namespace {

using tvk::gemm8::Shape;

// Row-major e4m3 [rows][K] as a 2-D tensor of bytes with 128 x box_rows boxes and the
// 128-byte swizzle (rows and columns past the end read as zeros).
bool make_map(CUtensorMap* map, const void* base, int rows, int K, int box_rows) {
  const tvk::gemm::EncodeTiled enc = tvk::gemm::encoder();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)K};
  const cuuint32_t box[2] = {(cuuint32_t)tvk::gemm8::kGroup, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box,
             estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
         CUDA_SUCCESS;
}

constexpr int kDevices = 64;
std::mutex g_mutex;
struct Device {
  int sms = 0, pairs = 0;   // CTAs and clusters of two that run at once
};
Device g_device[kDevices];

// Tile width: of the multiples of 32 (a chunk of 32 columns then lies in one block of
// weight scales), the one whose waves cover the fewest columns, each tile counted as
// `extra` columns wider for the H rows it loads again.
int tile_width(size_t m_tiles, int V, int units, int extra) {
  int best = tvk::gemm::kBN;
  long best_cost = 0;
  for (int bn = tvk::gemm::kBN; bn >= 128; bn -= 32) {
    const long tiles = (long)m_tiles * ((V + bn - 1) / bn);
    const long cost = (tiles + units - 1) / units * (bn + extra);
    if (best_cost == 0 || cost < best_cost) {
      best_cost = cost;
      best = bn;
    }
  }
  return best;
}

template <bool kPair, bool kStats>
cudaError_t launch(const CUtensorMap& map_h, const CUtensorMap& map_w, const float* h_scale,
                   const float* w_scale, int M, int V, int K, const Shape& shape, float c_hi,
                   float c_lo, void* logits, float2* part, int m_tiles, int n_tiles, int group,
                   int units, uint32_t* status, cudaStream_t stream) {
  using namespace tvk::gemm8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(std::min(m_tiles * n_tiles, units) * (kPair ? 2 : 1)), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kPair ? 1 : 0;
  const int store = V % 8 ? kStore2
                    : V % 16 == 0 && (reinterpret_cast<uintptr_t>(logits) & 31u) == 0 ? kStore32
                                                                                     : kStore16;
  return cudaLaunchKernelEx(&cfg, lm_head8_kernel<kPair, kStats>, map_h, map_w, h_scale, w_scale,
                            M, V, K, shape, c_hi, c_lo, static_cast<__nv_bfloat16*>(logits), part,
                            m_tiles, n_tiles, group, store, status);
}

template <bool kPair, bool kStats>
bool allow_smem() {
  return cudaFuncSetAttribute(tvk::gemm8::lm_head8_kernel<kPair, kStats>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)tvk::gemm8::kSmemBytes) == cudaSuccess;
}

// The current device's CTA and cluster counts, with the kernels' shared memory limits
// set; false on a CUDA error.
bool current_device(Device* out) {
  using namespace tvk::gemm8;
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= kDevices) return false;
  std::lock_guard<std::mutex> lock(g_mutex);
  Device& g = g_device[device];
  if (g.pairs < 1) {
    int sms = 0, pairs = 0;
    if (!allow_smem<false, false>() || !allow_smem<false, true>() || !allow_smem<true, false>() ||
        !allow_smem<true, true>() ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
      return false;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)sms / 2 * 2, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kSmemBytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&pairs, lm_head8_kernel<true, true>, &cfg) != cudaSuccess ||
        pairs < 1)
      return false;
    g.sms = sms;
    g.pairs = std::min(pairs, sms / 2);
  }
  *out = g;
  return true;
}

// One row tile: single SMs, bound by W's bytes; more: SM pairs.
bool pairs_for(size_t M) { return M > tvk::gemm::kBM; }

int width_for(size_t M, int V, const Device& g) {
  const bool pair = pairs_for(M);
  const size_t tile_rows = pair ? 2 * tvk::gemm::kBM : tvk::gemm::kBM;
  return tile_width((M + tile_rows - 1) / tile_rows, V, pair ? g.pairs : g.sms,
                    pair ? 256 : 64);
}

}  // namespace

size_t tv_lm_head_scaled_scratch(size_t rows, int V) {
  using tvk::gemm::kBM;
  Device g;
  if (!current_device(&g)) {
    cudaGetLastError();
    return 0;
  }
  rows = std::min<size_t>(rows, INT_MAX);
  size_t most = 0;
  for (size_t M = std::min<size_t>(rows, kBM);;
       M = std::min<size_t>(rows, (M / (2 * kBM) + 1) * 2 * kBM)) {
    const int bn = width_for(M, V, g);
    most = std::max(most, M * ((V + bn - 1) / bn));
    if (M >= rows) return most;
  }
}

int tv_launch_lm_head_scaled(const void* hidden, const float* hidden_scales, const void* weight,
                             const float* weight_scales, int M, int K, int V, float c_hi,
                             float c_lo, void* logits, float2* part, float2* row_stats,
                             uint32_t* status, cudaStream_t stream) {
  using namespace tvk::gemm8;
  if (M <= 0) return 0;
  Device g;
  if (!current_device(&g)) {
    cudaGetLastError();
    return -5;
  }
  const bool pair = pairs_for(M);
  const int tile_rows = pair ? 2 * kBM : kBM;
  const int units = pair ? g.pairs : g.sms;
  const int m_tiles = (M + tile_rows - 1) / tile_rows;
  Shape shape;
  shape.a_box = std::min(kBM, (M + 7) / 8 * 8);
  shape.bn = width_for(M, V, g);
  shape.stages = (int)std::min<size_t>(
      kMaxStages, kRingBytes / (shape.a_bytes() + shape.b_bytes(pair)));
  CUtensorMap map_h, map_w;
  if (!make_map(&map_h, hidden, M, K, shape.a_box) ||
      !make_map(&map_w, weight, V, K, pair ? shape.bn / 2 : shape.bn))
    return -5;
  const int n_tiles = (V + shape.bn - 1) / shape.bn;
  const int group = (int)std::max<size_t>(1, kGroupBytes / ((size_t)tile_rows * K));
  auto run = pair ? (row_stats ? launch<true, true> : launch<true, false>)
                  : (row_stats ? launch<false, true> : launch<false, false>);
  if (run(map_h, map_w, hidden_scales, weight_scales, M, V, K, shape, c_hi, c_lo, logits, part,
          m_tiles, n_tiles, group, units, status, stream) != cudaSuccess) {
    cudaGetLastError();
    return -5;
  }
  return row_stats ? tv_launch_merge(part, n_tiles, M, c_hi, c_lo, row_stats, stream) : 0;
}
