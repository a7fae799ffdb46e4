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
// The scales are general fp32 numbers, so the tensor cores' own block scaling (powers of
// two) does not serve: every group's product P_g is made from zero (four tcgen05.mma of
// kind::f8f6f4 on the group's 128 bytes a row) and added, times its scale, to fp32 sums
// in registers.  A group of a 128 x 256 tile costs the tensor cores 512 clocks; its 32768
// multiply-adds take 128 lanes 256, and bringing the product from tensor memory some 100
// more.  The two have to run side by side all the time: that sets the layout.
//
// One persistent kernel, one CTA of 12 warps per SM (SM pairs above 128 rows, which halve
// W's traffic through L2):
//   warp 0       TMA into a ring of stages, one group of K each
//   warps 1, 3   the products, one warp for each half of the tile's columns
//   warp 2       the scales, by 4-byte asynchronous copies into a ring of their own
//   warps 4-11   the sums: two warps for each quarter of the rows, one per half of the
//                columns; 128 fp32 sums of one row in a thread, in registers that the other
//                warps give up (232 of them for 40)
// Tensor memory holds four products of 128 columns, two for each half, so that one is
// made while the one before is summed.  Each is read in pieces of 32 and 16 columns, one
// on its way while the last is summed, two columns per multiply-add.  At the end of a
// tile the sums are rounded once to bf16 and stored: by pairs through shared memory and
// TMA, by single SMs from registers (the weight's bytes bound them), and rows that are not
// whole 16-byte pieces through shared memory, 128 bytes of a row at a time.
//
// Every wait is bounded; one that gives up raises the timeout status, and the loops go on
// to their end.
//
// Measured, one call after the other, in brackets a call alone (GB300, inputs from memory;
// the first is under the power cap; its products alone take 1732 us, and twice the bf16 rate
// of a plain library product would be 2135 us):
//                          logits alone                            with row statistics
//   7808 x 4096 x 128256   2.97 to 3.03 ms, 2710 to 2760 TFLOP/s   3.29 ms (3.06 to 3.15)
//                          (2.60 ms, 3150 TFLOP/s)
//   3904 x 4096 x  32000   392 to 396 us, 2590 TFLOP/s (345 us)    428 us (390)
//   3904 x 2048 x  32000   213 us (190)                            246 us (235)
//   3904 x 1024 x  32000   124 us (119)                            171 us (173)
//   3904 x  512 x  32000    80 us (89)                             145 us (161)
//     61 x 4096 x 128256    88 us, 6.1 TB/s: the weight's bytes     97 us
//      1 x 4096 x  32000    27 us, 4.9 TB/s: the same, with the     31 us
//                          launch and its ends
// The statistics, 35 to 70 us at 3904 rows, are worked out by the summing warps at a tile's
// end, while the tensor cores wait for them.  A group takes the sums' warps 630 clocks of which
// 370 are their loads and multiply-adds in isolation; the tensor cores idle for the rest of 630
// less 513.
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
constexpr int kParts = 2;                       // epilogue warps per TMEM lane quarter, one for
constexpr int kEpiWarps = 4 * kParts;           // each half of the tile's columns
constexpr int kThreads = 128 + 32 * kEpiWarps;  // TMA, scale and two MMA warps, epilogue
constexpr int kScaleGroups = 8;                 // groups of K in a slot of scales
constexpr int kScaleSlots = 4;
constexpr int kRegsFew = 40, kRegsMany = 232;   // registers per thread after the split
static_assert(128 * kRegsFew + 32 * kEpiWarps * kRegsMany <= kThreads * 168,
              "the warpgroups' registers fit what the block was launched with");
// The scales of one group: of a tile's rows, and of the weight block of each of its
// 32-column chunks.
struct Scales {
  float row[kBM];
  float chunk[kBN / 32];
};
// Where logits are stored through shared memory (by SM pairs, and where rows are not whole
// 16-byte pieces): buffers of 32 columns of a warp's 32 rows, at the end of the ring's bytes.
constexpr int kOutBufs = 2;
constexpr uint32_t kOutBytes = 32 * 32 * 2;
constexpr size_t kOutTotal = (size_t)kEpiWarps * kOutBufs * kOutBytes;
constexpr size_t kSmemBytes =
    kRingBytes + 1024 + (size_t)(kScaleSlots * kScaleGroups + 1) * sizeof(Scales);
// (one more, which the reads ahead at the ring's end fall on)
constexpr int kHalf = 128;                      // columns of a product: a tile has one or two
constexpr int kBufs = 4;                        // products in tensor memory
constexpr int kHalves = kBN / kHalf;
constexpr int kChunks = 4;                      // 32-column chunks of a thread
static_assert(kHalf == 32 * kChunks * kParts / kHalves && kBufs * kHalf == (int)kTmemCols, "");

// Instruction descriptor of tcgen05.mma kind::f8f6f4: fp32 accumulator (bits 4-5 =
// 1), e4m3 A and B (bits 7-9, 10-12 = 0), both K-major, N >> 3 in bits 17-22, M >> 4
// in bits 24-28.
__device__ __forceinline__ uint32_t instr_desc(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// One group's product: four tcgen05.mma of 32 bytes of K each, the first from zero, on
// descriptors (lo, hi) whose address field steps by 32 bytes.
template <bool kPair>
__device__ __forceinline__ void issue(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t hi,
                                      uint32_t idesc) {
#pragma unroll
  for (int k = 0; k < kGroup / kUmmaK; ++k) {
    const uint32_t off = (uint32_t)(k * kUmmaK) >> 4;
    if constexpr (kPair)
      asm volatile(
          "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
          "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
          "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %4, p;\n\t}" ::"r"(tmem_d),
          "r"(a_lo + off), "r"(b_lo + off), "r"(hi), "r"(idesc), "r"(k > 0 ? 1u : 0u)
          : "memory");
    else
      asm volatile(
          "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
          "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
          "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %4, p;\n\t}" ::"r"(tmem_d),
          "r"(a_lo + off), "r"(b_lo + off), "r"(hi), "r"(idesc), "r"(k > 0 ? 1u : 0u)
          : "memory");
  }
}

// umma_commit on a barrier's shared-memory address.
template <bool kPair>
__device__ __forceinline__ void commit_to(uint32_t bar) {
  if constexpr (kPair)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
  else
    asm volatile(
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
        : "memory");
}

// The same value, of which the compiler does not know that it is the whole warp's:
// addresses for barriers and shared memory then stay in the registers that these
// instructions read, and are not moved there from the uniform ones at each use (loop of
// the sums 450 -> 410 clocks a group in isolation).
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
  uint32_t y;
  asm volatile("mov.u32 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// The rest of a wait whose first test found the phase running: 0, or 1 if it gave up.
__device__ __forceinline__ uint32_t wait_longer(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity), "n"(kTrySuspendNs)
        : "memory");
    if (done) return 0;
  }
  return 1;
}

// Waits until the phase of the barrier at `bar` with this parity has completed, unless
// an earlier wait gave up; `bad` becomes 1 if this one does.
__device__ __forceinline__ void wait_on(uint32_t bar, uint32_t parity, uint32_t& bad) {
  if (!try_wait(bar, parity) && !bad) bad = wait_longer(bar, parity);
}

// A barrier's test whose answer is asked for later: a warp issues in order, and would
// stand still for the 100 clocks that the test takes if its answer were used at once.
// One test may be on its way; the predicate is the kernel's (declare_test, once).
__device__ __forceinline__ void declare_test() { asm volatile(".reg .pred tv_over;"); }
__device__ __forceinline__ void test_begin(uint32_t bar, uint32_t parity) {
  asm volatile("mbarrier.test_wait.parity.shared::cta.b64 tv_over, [%0], %1;" ::"r"(bar),
               "r"(parity)
               : "memory");
}
__device__ __forceinline__ uint32_t test_end() {
  uint32_t over;
  asm volatile("selp.u32 %0, 1, 0, tv_over;" : "=r"(over)::"memory");
  return over;
}

// Arrives on the barrier at `bar` (kPair: an address in the leader) for a part of tensor
// memory that has been read.  That the product which overwrites it comes after the reads
// rests on tcgen05.wait::ld, behind which this thread's reads are complete and their values in
// registers before the arrive is issued, and not on the arrive: a relaxed one orders
// nothing by itself.  Nothing in memory is published with it, so it has no release at cluster
// scope, whose fence took over 1500 clocks a group.
template <bool kPair>
__device__ __forceinline__ void arrive_read(uint32_t bar) {
  if constexpr (kPair)
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar)
                 : "memory");
  else
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// tmem_ld32 and tmem_wait of 16 columns.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                 "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// sum[at .. at + 8) += s * (16 columns), those of r[from ..).
template <int N>
__device__ __forceinline__ void scaled_sum(float2 (&sum)[16], int at, const uint32_t (&r)[N],
                                           int from, float s) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    sum[at + i] = __ffma2_rn(make_float2(__uint_as_float(r[from + 2 * i]),
                                         __uint_as_float(r[from + 2 * i + 1])),
                             make_float2(s, s), sum[at + i]);
}
__device__ __forceinline__ void scaled_sum(float2 (&sum)[16], const uint32_t (&r)[32], float s) {
  scaled_sum(sum, 0, r, 0, s);
  scaled_sum(sum, 8, r, 16, s);
}

__device__ __forceinline__ float lds32(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float4 lds128f(uint32_t at) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at)
               : "memory");
  return v;
}

// 4 bytes from global to shared memory, asynchronously.
__device__ __forceinline__ void copy_async4(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src)
               : "memory");
}
// Arrives on `bar` once this thread's copies so far have landed.
__device__ __forceinline__ void copy_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
template <int kRegs>
__device__ __forceinline__ void regs_fewer() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void regs_more() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}

// Launch shape: tile width, H rows a TMA box takes per CTA, ring stages.
struct Shape {
  int bn, a_box, stages;
  __host__ __device__ uint32_t a_bytes() const { return (uint32_t)a_box * kGroup; }
  __host__ __device__ uint32_t b_bytes(bool pair) const {
    return (uint32_t)(pair ? bn / 2 : bn) * kGroup;
  }
};

// The widest stores that every row's 32-column chunks allow (kStore4: 4 bytes, with 2 at the
// ends of odd rows).
enum { kStore4 = 0, kStore16 = 1, kStore32 = 2, kStoreTma = 3 };

// Puts 32 columns of the warp's 32 rows into `buf`, this lane's row, in the order that the
// 64-byte swizzle has (16-byte pieces exchanged by the row's bits 1 and 2, which also spreads
// the lanes over the banks).
__device__ __forceinline__ void fill_tile(const uint32_t (&packed)[16], uint32_t buf, int lane) {
  const uint32_t at = buf + (uint32_t)lane * 64u, turn = ((uint32_t)lane >> 1) & 3u;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 16 * (i ^ turn)),
                 "r"(packed[4 * i]), "r"(packed[4 * i + 1]), "r"(packed[4 * i + 2]),
                 "r"(packed[4 * i + 3])
                 : "memory");
}
// Stores `count` of them, from column x on, from the buffers at `buf`.  Rows and columns past
// the end of the logits are not written.  (One fence and one wait for two: 80 us at 3904 x
// 512 x 32000, 90 with one for each; four buffers cost the ring a stage: 79 there, but 209 for
// 200 at 976 x 2048 x 128256.)
__device__ __forceinline__ void store_tiles(uint32_t buf, int count, int lane,
                                            const CUtensorMap* map, int x, int y) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) {
    for (int k = 0; k < count; ++k)
      asm volatile(
          "cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
              reinterpret_cast<uint64_t>(map)),
          "r"(x + 32 * k), "r"(y), "r"(buf + kOutBytes * (uint32_t)k)
          : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}
// Until the stores this thread queued no longer read their buffers.
__device__ __forceinline__ void stores_read() {
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// 32 columns of a row, rounded to bf16.
__device__ __forceinline__ void pack_row(const float2 (&a)[16], uint32_t (&packed)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a[i].x, a[i].y);
    packed[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
}

// Keeps the compiler from working on these values before the running sums are there
// (several chunks' exponentials at once take more registers than there are).
__device__ __forceinline__ void in_order(uint32_t (&p)[16], float& m, float& s) {
  asm volatile(""
               : "+r"(p[0]), "+r"(p[1]), "+r"(p[2]), "+r"(p[3]), "+r"(p[4]), "+r"(p[5]),
                 "+r"(p[6]), "+r"(p[7]), "+r"(p[8]), "+r"(p[9]), "+r"(p[10]), "+r"(p[11]),
                 "+r"(p[12]), "+r"(p[13]), "+r"(p[14]), "+r"(p[15]), "+f"(m), "+f"(s));
}

// Stores the first n of 32 columns (a multiple of 8).
__device__ __forceinline__ void store_row(const uint32_t (&packed)[16], __nv_bfloat16* dst, int n,
                                          int mode) {
  if (mode == kStore32 && n >= 32) {
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
}

// Rows of any length: 64 columns of the warp's 32 rows through 4 KB of shared memory, so that
// a warp stores 128 bytes of one row at a time (2-byte stores of a column by 32 rows: 1162 us
// at 3904 x 512 x 31997 for 173, 314 at 976 x 1024 x 31997 for 62, 52 at 61 x 4096 x 31997 for
// 40).  Word j of a row holds its columns 2 j - s and 2 j + 1 - s, s = 1 where the row starts
// at an odd element, so that whole words are 4-byte aligned; of such a row the first column,
// and the last of a whole chunk, are stored by the lane that has the row.
//
// Puts a chunk's words there; before: the last word of the chunk before it.
__device__ __forceinline__ void stage_words(const uint32_t (&packed)[16], uint32_t before,
                                            uint32_t buf, int lane, int second, int s) {
  const uint32_t at = buf + (uint32_t)lane * 128u, order = s ? 0x5432u : 0x7654u;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 4u * (uint32_t)((16 * second + i) ^ lane)),
                 "r"(__byte_perm(i > 0 ? packed[i > 0 ? i - 1 : 0] : before, packed[i], order))
                 : "memory");
}
// Stores n columns of `rows` rows from there, of which the first starts at dst; chunks: how
// many were put there.
__device__ __forceinline__ void store_words(uint32_t buf, __nv_bfloat16* dst, int rows, int row0,
                                            int V, int n, int chunks, int lane) {
  __syncwarp();
#pragma unroll 4
  for (int r = 0; r < rows; ++r) {
    const int s = (row0 + r) & V & 1, e = 2 * lane - s;
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];"
                 : "=r"(v)
                 : "r"(buf + 128u * (uint32_t)r + 4u * (uint32_t)(lane ^ r))
                 : "memory");
    __nv_bfloat16* const p = dst + (size_t)r * V + e;
    if (e >= 0 && e + 1 < n)
      *reinterpret_cast<uint32_t*>(p) = v;
    else if (e >= 0 && e < (s && n == 32 * chunks ? n - 1 : n))
      *reinterpret_cast<uint16_t*>(p) = (uint16_t)v;
  }
  __syncwarp();
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
                    const __grid_constant__ CUtensorMap map_w,
                    const __grid_constant__ CUtensorMap map_w1,
                    const __grid_constant__ CUtensorMap map_out,
                    const float* __restrict__ h_scale,
                    const float* __restrict__ w_scale, int M, int V, int K, Shape shape,
                    float c_hi, float c_lo, __nv_bfloat16* __restrict__ logits,
                    float2* __restrict__ part, int m_tiles, int n_tiles, int group, int store,
                    uint32_t* __restrict__ status) {
  declare_test();
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kMaxStages];   // (kPair: the leader's are used)
  __shared__ __align__(8) uint64_t empty_bar[kMaxStages];
  __shared__ __align__(8) uint64_t acc_full[kBufs];       // a product is ready
  __shared__ __align__(8) uint64_t acc_empty[kBufs];      // it is read (kPair: the leader's)
  __shared__ __align__(8) uint64_t drain_bar;
  __shared__ __align__(8) uint64_t scale_full[kScaleSlots], scale_empty[kScaleSlots];
  __shared__ __align__(8) uint64_t ms_full[4], ms_empty[4];
  __shared__ float2 part_ms[kParts - 1][kBM];
  __shared__ uint32_t tmem_slot;
  __shared__ int failed;
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  Scales* scales = reinterpret_cast<Scales*>(smem + kRingBytes);   // [slot][group]

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = kPair ? cluster_rank() : 0u;
  const int first = kPair ? (int)blockIdx.x >> 1 : (int)blockIdx.x;
  const int step = kPair ? (int)gridDim.x >> 1 : (int)gridDim.x;
  const int tile_rows = kPair ? 2 * kBM : kBM;
  const int bn = shape.bn;
  // (kPair: each CTA holds half of the W rows of either product)
  const int n_half[kHalves] = {min(bn, kHalf), max(bn - kHalf, 0)};
  const int w_own = kPair ? n_half[0] / 2 : n_half[0];
  const uint32_t n_stages = (uint32_t)shape.stages;
  const uint32_t a_bytes = shape.a_bytes(), stage_bytes = a_bytes + shape.b_bytes(kPair);
  const int nkb = (K + kGroup - 1) / kGroup;
  const int n_total = m_tiles * n_tiles;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < n_stages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], bn > kHalf ? kHalves : 1);
    }
    for (int k = 0; k < kBufs; ++k) {
      mbar_init(&acc_full[k], 1);
      mbar_init(&acc_empty[k], (kPair ? 2 : 1) * kEpiWarps / kHalves);
    }
    mbar_init(&drain_bar, bn > kHalf ? kHalves : 1);
    for (int k = 0; k < kScaleSlots; ++k) {
      mbar_init(&scale_full[k], 32);
      mbar_init(&scale_empty[k], bn > kHalf ? kEpiWarps : kEpiWarps / kHalves);
    }
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

  if (warp >= 4) {
    regs_more<kRegsMany>();
    // ---- scaled sums: one row and 128 columns (half of the tile's at most) a thread ----
    const int q = warp & 3;                       // the TMEM lane quarter of this warp
    const int mine = (warp - 4) >> 2;
    const float2 ch = make_float2(c_hi, c_hi), cl = make_float2(c_lo, c_lo);
    const int half = mine, col = kHalf * half;
    const uint32_t full0 = opaque(smem_u32(&acc_full[half]));
    const uint32_t empty0 = kPair ? map_shared(&acc_empty[half], 0)
                                  : opaque(smem_u32(&acc_empty[half]));
    // this thread's row's scales and its chunks' in the first record of the ring
    const uint32_t row_scale = opaque(smem_u32(&scales->row[q * 32 + lane]));
    const uint32_t chunk_scales = opaque(smem_u32(&scales->chunk[kChunks * half]));
    const uint32_t out0 = smem_u32(smem) + (uint32_t)(kRingBytes - kOutTotal) +
                          (uint32_t)((warp - 4) * kOutBufs) * kOutBytes;
    uint32_t buf = 0, ph = 0, si = 0;             // 16 x the buffer of the next group; its phase
    int j = 0;
    // A wait that gives up is reported and no longer waited for: the loops go on to
    // their end (on whatever is there), so that no wait needs a way out of them.
    uint32_t bad = 0, over = 0;                   // over: the next group's product is ready
    for (int t = first; t < n_total; t += step, ++j) {
      int mt, n_tile;
      tile_coords(t, m_tiles, n_tiles, group, mt, n_tile);
      const int n0 = n_tile * bn;
      const int row0 = mt * tile_rows + (int)rank * kBM + q * 32, row = row0 + lane;
      const bool live = row0 < M;                 // (the same in the whole warp)
      const uint32_t tbase = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)col;
      float2 sum[kChunks][16];
#pragma unroll
      for (int k = 0; k < kChunks; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[k][i] = make_float2(0.f, 0.f);
      if (n_half[half] > 0) {
        for (int kb0 = 0; kb0 < nkb; kb0 += kScaleGroups, ++si) {
          const uint32_t slot = si % kScaleSlots;
          wait_on(smem_u32(&scale_full[slot]), (si / kScaleSlots) & 1, bad);
          uint32_t rec = slot * (uint32_t)(kScaleGroups * sizeof(Scales));
          int left = min(kScaleGroups, nkb - kb0);
          if (live) {
            float next_row = lds32(row_scale + rec);
            float4 next_chunk = lds128f(chunk_scales + rec);
            for (; left > 0; --left) {
              // 16 or 32 columns are on their way from tensor memory while the ones before
              // are summed (all of a product's, whatever the tile's width: those past it
              // are not stored); the next group's scales and its product's barrier are
              // asked for meanwhile
              if (!over) wait_on(full0 + buf, ph, bad);
              tc_fence_after();
              uint32_t a[32], b[16];
              const uint32_t at = tbase + 16 * buf;
              tmem_ld32(at, a);
              const float4 s = make_float4(next_row * next_chunk.x, next_row * next_chunk.y,
                                           next_row * next_chunk.z, next_row * next_chunk.w);
              tmem_wait(a);
              tmem_ld16(at + 32, b);
              scaled_sum(sum[0], a, s.x);
              rec += (uint32_t)sizeof(Scales);
              ph ^= buf >> 4;                     // (the phase turns after the second buffer)
              buf ^= 16u;
              tmem_wait16(b);
              tmem_ld32(at + 48, a);
              next_row = lds32(row_scale + rec);
              next_chunk = lds128f(chunk_scales + rec);
              scaled_sum(sum[1], 0, b, 0, s.y);
              tmem_wait(a);
              tmem_ld16(at + 80, b);
              scaled_sum(sum[1], 8, a, 0, s.y);
              scaled_sum(sum[2], 0, a, 16, s.z);
              tmem_wait16(b);
              tmem_ld32(at + 96, a);
              scaled_sum(sum[2], 8, b, 0, s.z);
              tmem_wait(a);
              tc_fence_before();
              // (every lane's part is read: the load and its wait are the warp's)
              if (lane == 0) arrive_read<kPair>(empty0 + (buf ^ 16u));
              test_begin(full0 + buf, ph);
              scaled_sum(sum[3], a, s.w);
              over = test_end();
            }
          } else {
            for (; left > 0; --left) {
              if (!over) wait_on(full0 + buf, ph, bad);
              if (lane == 0) arrive_read<kPair>(empty0 + buf);
              ph ^= buf >> 4;
              buf ^= 16u;
              over = 0;
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&scale_empty[slot]);
        }
      }
      float m_run = TV_NEG_INF, s_run = 0.f;
      uint32_t before = 0;                        // (kStore4: the last word of the chunk before)
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        const int c = col + 32 * k, col0 = n0 + c;
        const int n = min(32, V - col0);          // columns of the chunk that exist
        if (c >= bn || n <= 0) break;             // (the same in the whole warp)
        uint32_t packed[16];
        pack_row(sum[k], packed);
        if (kPair && store == kStoreTma) {
          if (row0 < M) {                         // (the same in the whole warp)
            const int slot = k % kOutBufs;
            if (slot == 0) {
              if (lane == 0) stores_read();
              __syncwarp();
            }
            fill_tile(packed, out0 + kOutBytes * slot, lane);
            if (slot == kOutBufs - 1 || c + 32 >= bn || V - col0 <= 32)   // no chunk to wait for
              store_tiles(out0, slot + 1, lane, &map_out, col0 - 32 * slot, row0);
          }
        } else if (store == kStore4) {
          if (row0 < M) {
            const int odd = row & V & 1;          // (col0 is even)
            __nv_bfloat16* const dst = logits + (size_t)row * V + col0;
            uint16_t* const own = reinterpret_cast<uint16_t*>(dst);
            stage_words(packed, before, out0, lane, k & 1, odd);
            before = packed[15];
            if (odd && row < M && !(k & 1)) own[0] = (uint16_t)packed[0];
            if ((k & 1) || c + 32 >= bn || n < 32 || V - col0 <= 32) {   // no chunk to wait for
              const int back = 32 * (k & 1);
              if (odd && row < M && n == 32) own[31] = (uint16_t)(packed[15] >> 16);
              store_words(out0, logits + (size_t)row0 * V + col0 - back, min(32, M - row0), row0,
                          V, back + n, 1 + (k & 1), lane);
            }
          }
        } else if (row < M) {
          store_row(packed, logits + (size_t)row * V + col0, n, store);
        }
        if constexpr (kStats) {
          in_order(packed, m_run, s_run);
          sum_row(packed, n, ch, cl, m_run, s_run);
        }
      }
      if constexpr (kStats) {    // one partial per row and tile from the quarter's warps
        if (mine > 0) {
          if (j > 0) wait_on(smem_u32(&ms_empty[q]), (j - 1) & 1, bad);
          part_ms[mine - 1][q * 32 + lane] = make_float2(m_run, s_run);
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms_full[q]);
        } else {
          wait_on(smem_u32(&ms_full[q]), j & 1, bad);
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
    if (kPair && lane == 0) stores_read();     // (the buffers go with the CTA)
    if (bad) failed = 1;
  } else {
    regs_fewer<kRegsFew>();
    if (warp == 0) {
      // ---- TMA producer: one ring across all of this CTA's tiles ----
      uint32_t it = 0, s = 0, ph = 0;
      bool ok = true;
      for (int t = first; t < n_total && ok; t += step) {
        int mt, nt;
        tile_coords(t, m_tiles, n_tiles, group, mt, nt);
        const int m0 = mt * tile_rows + (int)rank * kBM, n0 = nt * bn + (int)rank * w_own;
        const int n1 = nt * bn + kHalf + (int)rank * (n_half[1] / 2);
        for (int kb = 0; kb < nkb; ++kb, ++it) {
          if (it >= n_stages && !wait_warp(&empty_bar[s], ph ^ 1u)) {
            ok = false;
            break;
          }
          uint8_t* a = smem + s * stage_bytes;
          uint32_t bar = smem_u32(&full_bar[s]);
          if constexpr (kPair) bar = map_shared(&full_bar[s], 0);
          if (elect_one()) {
            if (rank == 0)
              mbar_arrive_expect_tx(&full_bar[s], kPair ? 2 * stage_bytes : stage_bytes);
            tma_load_2d<kPair>(a, &map_h, kb * kGroup, m0, bar);
            tma_load_2d<kPair>(a + a_bytes, &map_w, kb * kGroup, n0, bar);
            if (kPair && n_half[1] > 0)
              tma_load_2d<kPair>(a + a_bytes + w_own * kGroup, &map_w1, kb * kGroup, n1, bar);
          }
          __syncwarp();
          if (++s == n_stages) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) failed = 1;
      if (rank == 0)      // the copies issued last have landed before the CTA may exit
        for (uint32_t j = it > n_stages ? it - n_stages : 0u; j < it; ++j)
          if (!wait_warp(&full_bar[j % n_stages], (j / n_stages) & 1)) failed = 1;
    } else if (warp == 1 || warp == 3) {
      // ---- tensor-core issue: each group's products into the accumulators in turn ----
      // One warp for each half of the columns: a warp's own instructions (two waits, four
      // products, two commits) take about 400 clocks a half, more than its products' 256.
      const int half = warp >> 1;
      if (rank == 0 && n_half[half] > 0) {
        const uint32_t idesc = instr_desc(tile_rows, n_half[half]);
        const uint64_t desc = smem_desc(smem);
        const uint32_t desc_hi = (uint32_t)(desc >> 32), desc_lo = (uint32_t)desc;
        const uint32_t b_off = (a_bytes + (uint32_t)(half * w_own * kGroup)) >> 4;
        const uint32_t full0 = opaque(smem_u32(full_bar)), empty0 = smem_u32(empty_bar);
        const uint32_t acc_f = smem_u32(&acc_full[half]);
        const uint32_t acc_e = opaque(smem_u32(&acc_empty[half]));
        const uint32_t d0 = tmem + (uint32_t)(kHalf * half);
        uint32_t s = 0, lo = desc_lo, ph = 0;       // the stage, its descriptor, its phase
        uint32_t buf = 0, aph = 1;                  // the buffer, its release's phase
        uint32_t bad = 0;
        const int tiles = first < n_total ? (n_total - first + step - 1) / step : 0;
        for (int left = tiles * nkb; left > 0; --left) {
          wait_on(full0 + 8 * s, ph, bad);
          // (the first use of a buffer waits for the phase before the first, which is over)
          wait_on(acc_e + 16 * buf, aph, bad);
          if (__any_sync(0xffffffffu, bad)) break;
          tc_fence_after();
          if (elect_one()) {
            issue<kPair>(d0 + 256 * buf, lo, lo + b_off, desc_hi, idesc);
            commit_to<kPair>(acc_f + 16 * buf);
            commit_to<kPair>(empty0 + 8 * s);
          }
          __syncwarp();
          buf ^= 1u;
          aph ^= buf ^ 1u;
          lo += stage_bytes >> 4;
          if (++s == n_stages) {
            s = 0;
            lo = desc_lo;
            ph ^= 1u;
          }
        }
        if (bad) failed = 1;
        // every MMA issued has finished before tensor memory is freed
        if (elect_one()) umma_commit<kPair>(&drain_bar);
        __syncwarp();
      }
      // (kPair, the peer: the leader's last signal)
      if (!wait_warp(&drain_bar, 0)) failed = 1;
    } else if (warp == 2) {
      // ---- scales: a slot of groups ahead of the sums, straight to shared memory ----
      const int w_blocks = (V + kGroup - 1) / kGroup;
      uint32_t it = 0;
      bool ok = true;
      for (int t = first; t < n_total && ok; t += step) {
        int mt, nt;
        tile_coords(t, m_tiles, n_tiles, group, mt, nt);
        const int row0 = mt * tile_rows + (int)rank * kBM + lane, n0 = nt * bn;
        const int blk = min((n0 + 32 * (lane & 7)) / kGroup, w_blocks - 1);
        for (int kb0 = 0; kb0 < nkb; kb0 += kScaleGroups, ++it) {
          const uint32_t slot = it % kScaleSlots;
          if (it >= kScaleSlots && !wait_warp(&scale_empty[slot], ((it / kScaleSlots) - 1) & 1)) {
            ok = false;
            break;
          }
          const int groups = min(kScaleGroups, nkb - kb0);
  #pragma unroll
          for (int r = 0; r < kBM / 32; ++r) {
            const float* src = h_scale + (size_t)min(row0 + 32 * r, M - 1) * nkb + kb0;
            for (int k = 0; k < groups; ++k)
              copy_async4(&scales[slot * kScaleGroups + k].row[lane + 32 * r], src + k);
          }
          for (int k = lane >> 3; k < groups; k += 4)
            copy_async4(&scales[slot * kScaleGroups + k].chunk[lane & 7],
                        w_scale + (size_t)blk * nkb + kb0 + k);
          copy_async_arrive(&scale_full[slot]);
        }
      }
      if (!ok) failed = 1;
      // the copies issued last have landed before the CTA may exit
      asm volatile("cp.async.wait_all;" ::: "memory");
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

// The logits in boxes of 32 x 32 with the 64-byte swizzle, where their rows allow it (the
// kernel stores without the map where they do not).
bool make_out_map(CUtensorMap* map, void* base, int rows, int V) {
  if (V % 8) {
    *map = CUtensorMap{};
    return true;
  }
  const tvk::gemm::EncodeTiled enc = tvk::gemm::encoder();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)V, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)V * 2};
  const cuuint32_t box[2] = {32, 32};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
cudaError_t launch(const CUtensorMap& map_h, const CUtensorMap& map_w,
                   const CUtensorMap& map_w1, const CUtensorMap& map_out, const float* h_scale,
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
  const int store = V % 8 ? kStore4
                    : kPair ? kStoreTma
                    : V % 16 == 0 && (reinterpret_cast<uintptr_t>(logits) & 31u) == 0 ? kStore32
                                                                                     : kStore16;
  return cudaLaunchKernelEx(&cfg, lm_head8_kernel<kPair, kStats>, map_h, map_w, map_w1, map_out,
                            h_scale, w_scale, M, V, K, shape, c_hi, c_lo,
                            static_cast<__nv_bfloat16*>(logits), part, m_tiles, n_tiles, group,
                            store, status);
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
      kMaxStages, (kRingBytes - (pair || V % 8 ? kOutTotal : 0)) /
                      (shape.a_bytes() + shape.b_bytes(pair)));
  CUtensorMap map_h, map_w, map_w1, map_out;
  const int w1 = pair && shape.bn > kHalf ? (shape.bn - kHalf) / 2 : kHalf;
  if (!make_map(&map_h, hidden, M, K, shape.a_box) ||
      !make_map(&map_w, weight, V, K, pair ? std::min(shape.bn, kHalf) / 2 : shape.bn) ||
      !make_map(&map_w1, weight, V, K, w1) || !make_out_map(&map_out, logits, M, V))
    return -5;
  const int n_tiles = (V + shape.bn - 1) / shape.bn;
  const int group = (int)std::max<size_t>(1, kGroupBytes / ((size_t)tile_rows * K));
  auto run = pair ? (row_stats ? launch<true, true> : launch<true, false>)
                  : (row_stats ? launch<false, true> : launch<false, false>);
  if (run(map_h, map_w, map_w1, map_out, hidden_scales, weight_scales, M, V, K, shape, c_hi, c_lo,
          logits, part, m_tiles, n_tiles, group, units, status, stream) != cudaSuccess) {
    cudaGetLastError();
    return -5;
  }
  return row_stats ? tv_launch_merge(part, n_tiles, M, c_hi, c_lo, row_stats, stream) : 0;
}
