// dard_experts.cu - dard_experts: the products of a mixture of experts, grouped over the
// (token, slot) pairs that dard_route sorted by expert.
//
//   gather_rows      many rows: x in the plan's order
//   product<.., 1>   h = silu(w1 x) * (w3 x) of every pair, rounded (MXFP8 or bf16)
//   product<.., 2>   o = w2 h of every pair
//   combine          y_t = sum over the slots of token t of weight * o
//
// Both products are one persistent tcgen05 kernel. An output tile is the pairs of one expert (the
// rows of A) by kN weight rows (B, N = kN); what a CTA computes follows from `offsets` alone,
// so no size of an expert ever travels to the host. In phase 1 half of a tile's weight rows are
// w1's and half the same rows of w3, so that the gate and the value it scales meet in one
// thread's registers: a thread of the epilogue holds one pair (TMEM lane) and 32 consecutive
// hidden elements, which is one MX block: its scale needs no exchange.
//
// Three variants, chosen by the call's sizes (make_plan):
//   pairs   two CTAs of a cluster (cta_group::2) share one M = 256, N = 256 MMA: each holds 128
//           rows of A and 128 weight rows. A stage moves 32 KB into each SM's shared memory; one
//           CTA with a 128 x 256 tile would move 48 KB, which together with what the MMA reads is
//           more than shared memory carries (phase 1 at 2.3 against 2.9 PFLOP/s);
//   single  one CTA, M = 128, N = 128: more and smaller tiles, for calls with few rows;
//   few     at most 32 tokens: the same with a short A stage and deeper staging of the weights,
//           and no launch for the sum over the slots: a column tile's last CTA adds them up.
//
// Roles per CTA (warps: pairs 12, single 8, few 7):
//   epilogue    8 warps (single, few: 4): TMEM -> registers, then the accumulator is free for the
//               next tile while SwiGLU, the rounding and the stores run from registers;
//   producer    TMA: rows of A that lie side by side, weights, scales (cp.async.bulk). Pairs: each
//               rank fills its own shared memory, and both ranks' copies report to rank 0's
//               barriers, where the issuer waits. (A warp of rank 1 that waits for its copies and
//               tells rank 0 has to do so with release at cluster scope, at some 1500 cycles per
//               stage: 800 rows of 4096 x 12288 300 us instead of 114.);
//   issuer      TMEM allocation; scale copies (tcgen05.cp) and MMAs (pairs: in rank 0);
//   gather      single and few, phase 1: the rows of x by token (cp.async, 16 bytes per lane,
//               straight into the swizzled layout) and their scales.
//   Stage: 128 bytes of K of the A rows and of the weight rows (128-byte swizzle), plus scales.
//   TMEM: the accumulator, then the scales of two stages.
//
// Pairs read rows of x that an earlier launch (gather_rows) has put in the plan's order. For 4096
// rows of one expert of 4096 x 12288 the call took 378 us that way (372 now); with the rows gathered in
// phase 1 by cp.async from four warps 478, by TMA's row gather (tile::gather4) from four warps 448.
// For few rows the copy's launch costs more than the gather does.
//
// What bounds it, on GB300: pairs, 3.27 PFLOP/s in MXFP8 at 4096 x 4096 x 12288, the tensor pipe
// and shared memory together (with half of the weights' bytes left out it is 10 % faster, without
// its stores 7 %); 8192 tokens x 8 of 64 experts of 4096 x 2048 1.5-1.65 ms (the clock
// falls to 1500-1800 MHz at the power limit), of which gather_rows takes 75 us and combine 255 us, both
// HBM's bytes. Few: the weights' bytes (32 tokens x 8 of 64 of 2048 x 1024, 400 MB: 85 us where the
// experts have as many rows each, with no MMA at all 80; 90-93 where some have more) and for one
// token the chain of latencies (21.8 us for the two launches; its 52 MB alone would take 7.6).
// bf16, with twice the weights' bytes and half the tensor rate: one token 27-32 us, 32 tokens 141
// (5.6 TB/s), 1111 tokens x 6 of 40 of 2208 x 736 123, 800 rows of 4096 x 12288 184 (1.31 PFLOP/s),
// 8192 tokens x 8 of 64 of 4096 x 2048 2.46-2.56 ms (1.3 PFLOP/s).
//
// Every wait is bounded; one that gives up sets DARD_STATUS_TIMEOUT and the abort flag of its CTA
// (of both of a pair), on which every role leaves its loop. The producer (for a pair, rank 0's)
// then waits (bounded) for copies in flight and the issuer for its MMAs before shared memory and
// TMEM are released.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <type_traits>

#include "dard_host.cuh"
#include "dard_internal.h"
#include "dard_mx.cuh"
#include "dard_ptx.cuh"

namespace dard {
namespace {

constexpr int kTileM = 128;            // rows of A per CTA
constexpr int kTileB = 128;            // weight rows per CTA
constexpr int kStageK = 128;           // bytes of K per stage
constexpr int kMaxStages = 6;
constexpr int kGatherLag = 2;          // stages a gather warp has in flight
constexpr uint32_t kBytesB = kTileB * kStageK;
constexpr uint32_t kScaleBytes = 3 * kMxTileBytes;  // of a stage: A's, then two tiles of B's
constexpr int kGroupM = 16;            // row tiles that share a pass over an expert's columns
constexpr uint16_t kBothCtas = 0x3;

// The variants (see the top of the file). A CTA of the last two takes half of an SM's registers,
// shared memory and TMEM, so that the next launch's CTAs, which do not depend on this one for
// their weights, can sit next to it.
constexpr int kPairs = 0, kSingle = 1, kFew = 2;
constexpr int kFewTokens = 32;
template <int kVariant>
struct Shape {
  static constexpr bool kPair = kVariant == kPairs;
  static constexpr int kCtas = kPair ? 2 : 1;  // that share an MMA
  static constexpr int kStages = kPair ? 6 : kVariant == kSingle ? 3 : 5;
  // Rows of A that a stage holds, and of a row tile. The MMA reads 128: what lies behind (this
  // stage's B) gives rows of the accumulator that nobody reads. (An expert has more rows than
  // there are tokens where tokens name it in several slots: it then has several tiles.)
  static constexpr int kRowsA = kVariant == kFew ? kFewTokens : kTileM;
  static constexpr int kBoxA = kPair ? kTileM : 32;  // rows per copy
  static constexpr uint32_t kBytesA = kRowsA * kStageK, kStageBytes = kBytesA + kBytesB;
  static constexpr int kEpilogueWarps = kPair ? 8 : 4;
  static constexpr int kGatherWarps = kVariant == kFew ? 1 : 2;
  static constexpr int kProducerWarp = kEpilogueWarps, kIssueWarp = kProducerWarp + 1,
                       kGatherWarp = kIssueWarp + 1;
  static constexpr int kThreads = 32 * (kGatherWarp + kGatherWarps);
  static constexpr uint32_t kTmem = kPair ? 512 : 256;
  static constexpr uint32_t kScaleCol = kPair ? 256 : 128;  // first TMEM column of the scales
  static constexpr int kCtasPerSm = kPair ? 1 : 2;
};

struct ExpertsParams {
  const int32_t* offsets;
  const int32_t* rows;
  const int32_t* ids;
  const float* weights;
  const void* x;
  const uint8_t* x_scale;
  const uint8_t* scale_b[2];  // phase 1: w1, w3; phase 2: w2
  const uint8_t* a_scale;     // of the rows TMA reads (x in the plan's order, or h), in tiles
  uint8_t* xg;                // [row tiles * 128][dim]: x in the plan's order
  uint8_t* xg_scale;          // [row tiles][ceil(dim / 128)][512]
  uint8_t* h;                 // [row tiles * 128][hidden]
  uint8_t* h_scale;           // [row tiles][ceil(hidden / 128)][512]
  int32_t* arrived;           // few: per column tile of phase 2, the tiles done
  float* partial;             // [splits][pairs][dim]
  void* y;
  uint32_t* status;
  int64_t x_stride_bytes, x_scale_stride, y_stride;
  long long wait_cycles;
  int32_t tokens, experts, top_k, dim, hidden, pairs;
  int32_t k_elems, n_elems;     // of this phase: reduced length, weight rows per expert
  int32_t n_tiles;              // tiles over n_elems
  int32_t k_stages;             // stages over k_elems
  int32_t splits, split_stages; // phase 2: the reduction in `splits` runs of split_stages
  int32_t max_row_tiles;        // rows of the workspace / kTileM
  int32_t gather_shift;         // gather_rows: 1 << gather_shift warps per pair
  int32_t y_f32;
  int32_t direct;               // phase 2 writes y itself (top_k 1, one split)
  int32_t test_drop;            // test hook: the stage use whose B copy is never issued
};

// ---------------------------------------------------------------- PTX of this file
__device__ __forceinline__ void tma_load_3d(void* dst, const void* desc, uint64_t* bar, int32_t c0,
                                            int32_t c1, int32_t c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(desc)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// CTA pairs: tiled loads into the own shared memory that report to a barrier of either CTA of the
// pair, given by its shared::cluster address (with release at cluster scope).
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const void* desc, uint32_t bar, int32_t c0,
                                                 int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(desc)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const void* desc, uint32_t bar, int32_t c0,
                                                 int32_t c1, int32_t c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(desc)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}
// One 512-byte tile of scales (32 rows of 16 bytes) into four TMEM columns of every lane quarter;
// with kPair in both CTAs, each from its own shared memory.
template <bool kPair>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if constexpr (kPair)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
                 : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
                 : "memory");
}
template <bool kPair>
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if constexpr (kPair)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::
            "r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::
            "r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
        : "memory");
}
__device__ __forceinline__ void mma_ss_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Waits on a barrier, or looks at it, at the scope of what arrives there: the CTA, or (kPair) the
// cluster, whose other CTA arrives too.
template <bool kPair>
__device__ __forceinline__ bool try_wait(uint64_t* bar, uint32_t parity) {
  if constexpr (!kPair) return mbar_try_wait(bar, parity);
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Whether the phase with this parity has completed, without waiting.
template <bool kPair>
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  if constexpr (kPair)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  return ok != 0;
}
// CTA pairs: arrivals on a barrier of rank 0, given by its shared::cluster address. Relaxed: what
// they hand over is ordered by the tcgen05 fences around them (the accumulator), or is the
// number of bytes that copies will report to the barrier by themselves.
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_expect_tx_cluster(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar),
               "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void store_cluster(uint32_t addr, int32_t v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// mbar_wait that also gives up, once it has to wait, when the CTA's abort flag is set.
template <bool kPair>
__device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, long long limit,
                                       const volatile int32_t* abort_flag) {
  const long long t0 = clock64();
  while (!try_wait<kPair>(bar, parity)) {
    if (*abort_flag != 0 || clock64() - t0 > limit) return false;
  }
  return true;
}
// A place in the ring of stages, and the parity of its barriers' phase there: full[b] completes
// phase `phase` when stage b's copies have landed, empty[b] when they have been read. (On a new
// barrier the phase before the first counts as complete.)
struct Ring {
  int b = 0;
  uint32_t phase = 0;
  template <int kStages>
  __device__ __forceinline__ void next() {
    if (++b == kStages) {
      b = 0;
      phase ^= 1;
    }
  }
};
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}
template <int kPending>
__device__ __forceinline__ void cp_async_wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}
// 16 bytes that no one writes, read here (a plain load may be moved down to where it is used).
__device__ __forceinline__ uint4 load16_here(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
// 32 bytes to a 32-byte aligned address.
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]),
               "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// Unswizzled descriptor of a 32 x 16-byte tile of scales: eight-row groups 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128 >> 4) << 32) |
         (1ull << 46);
}
// Instruction descriptor of kind::mxf8f6f4: e4m3 operands, e8m0 scales; `ks` picks the scale
// byte of both operands (the K step within a stage).
__host__ __device__ constexpr uint32_t idesc_mx(uint32_t M, uint32_t N, uint32_t ks) {
  return (ks << 4) | ((N >> 3) << 17) | (1u << 23) | ((M >> 4) << 24) | (ks << 29);
}

struct __align__(16) Ctl {
  uint64_t full[kMaxStages], empty[kMaxStages];  // (pairs: rank 0's full is both CTAs')
  uint64_t acc_full, acc_free;
  uint64_t drained;  // every MMA the issuer launched has completed
  uint32_t tmem_base;
  int32_t abort;     // (pairs: set in both CTAs)
  int32_t last;      // few: this CTA's tile was its columns' last
  int32_t uses[2];   // pairs: stages that each rank has filled (both CTAs hold both)
  int32_t first_row[DARD_MAX_EXPERTS + 1];   // offsets, clamped to [0, pairs]
  int32_t first_tile[DARD_MAX_EXPERTS + 1];  // row tiles of the experts before
  // (pairs: after this, the same in units of two row tiles)
};

template <int kVariant>
constexpr size_t smem_bytes() {
  using S = Shape<kVariant>;
  return 1024 + static_cast<size_t>(S::kStages) * (S::kStageBytes + kScaleBytes) + sizeof(Ctl) +
         (S::kPair ? sizeof(int32_t) * (DARD_MAX_EXPERTS + 1) : 0);
}

// A CTA's part of one tile: rows [row, row + count) (count <= 0: none) of expert e, in row tile
// row_tile of h (kTileM rows apart, whatever the rows of a tile); column tile n, reduction split.
struct Tile {
  int e, row, count, row_tile, n, split;
};

// Tile `w` of the call. Within an expert, a group of row units takes each column tile in turn,
// so that CTAs that run together share weights and rows in L2. `e` walks forward.
template <int kVariant>
__device__ __forceinline__ bool get_tile(const ExpertsParams& p, const Ctl& c,
                                         const int32_t* first_unit, int rank, int64_t w, int& e,
                                         Tile& t) {
  constexpr int kUnitTiles = Shape<kVariant>::kCtas, kGroup = kGroupM / kUnitTiles;
  constexpr int kRows = Shape<kVariant>::kRowsA;
  const int per_unit = p.n_tiles * p.splits;
  if (w >= static_cast<int64_t>(first_unit[p.experts]) * per_unit) return false;
  while (w >= static_cast<int64_t>(first_unit[e + 1]) * per_unit) ++e;
  const int units = first_unit[e + 1] - first_unit[e];
  const int local = static_cast<int>(w - static_cast<int64_t>(first_unit[e]) * per_unit);
  const int group = local / (kGroup * per_unit);
  const int in_group = min(kGroup, units - group * kGroup);
  const int rest = local - group * kGroup * per_unit;
  const int m = (group * kGroup + rest % in_group) * kUnitTiles + rank;
  const int col = rest / in_group;
  t.e = e;
  t.n = col % p.n_tiles;
  t.split = col / p.n_tiles;
  t.row = c.first_row[e] + m * kRows;
  t.row_tile = c.first_tile[e] + m;
  // (a plan cut short at the workspace's end may leave a pair's second row tile outside)
  t.count = t.row_tile < c.first_tile[e + 1] ? min(kRows, c.first_row[e + 1] - t.row) : 0;
  return true;
}

// The plan's offsets, clamped to [0, pairs], and by expert the row tiles (kRows rows) and the units of
// kCtas row tiles before it, by the whole CTA. A plan that is none (offsets that fall) never
// reaches past the workspace. Ends without a barrier.
template <int kCtas, int kRows>
__device__ __forceinline__ void read_plan(const ExpertsParams& p, int32_t* first_row,
                                          int32_t* first_tile, int32_t* first_unit) {
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i <= p.experts; i += blockDim.x)
    first_row[i] = min(max(p.offsets[i], 0), p.pairs);
  __syncthreads();
  if (threadIdx.x >= 32) return;
  int carry_t = 0, carry_u = 0;
  for (int b = 0; b < p.experts; b += 32) {
    const int i = b + lane;
    const int n = i < p.experts ? max(first_row[i + 1] - first_row[i], 0) : 0;
    int tiles = (n + kRows - 1) / kRows;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, tiles, o);
      if (lane >= o) tiles += y;
    }
    const int end = min(carry_t + tiles, p.max_row_tiles);
    const int before = __shfl_up_sync(0xffffffffu, end, 1);
    const int start = lane == 0 ? carry_t : before;
    int units = (end - start + kCtas - 1) / kCtas;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, units, o);
      if (lane >= o) units += y;
    }
    if (i < p.experts) {
      first_tile[i + 1] = end;
      first_unit[i + 1] = carry_u + units;
    }
    carry_t = __shfl_sync(0xffffffffu, end, 31);
    carry_u += __shfl_sync(0xffffffffu, units, 31);
  }
  if (lane == 0) first_tile[0] = first_unit[0] = 0;
}

// Uses of r stay behind this point.
__device__ __forceinline__ void pin32(uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]),
                      "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}

// g / (1 + exp(-g)) by the hardware's exponential and division: off by about 2 + 1.2 |g| units in
// fp32's last place, and 0 below g = -87, where it is less than 2^-118. h is rounded to 8 bits (bf16)
// or 4 right after. With expf one token takes 23.7 us instead of 23.0 and 800 rows of 4096 x 12288
// 119.3 instead of 117.5; with expf and an IEEE division 43 and 130.
__device__ __forceinline__ float silu(float g) { return __fdividef(g, 1.f + __expf(-g)); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// AND of `ok` over the epilogue's warps, which it also syncs (so that they leave a loop together).
template <int kWarps>
__device__ __forceinline__ bool epilogue_and(bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(ok)), "n"(32 * kWarps)
      : "memory");
  return r != 0;
}

// Columns col .. col + 3 of y_t = sum over slots (in order) of weight * (sum over splits of the
// pair's product). The products of up to eight slots are in flight at once.
__device__ __forceinline__ void combine_columns(const ExpertsParams& p, int64_t t, int col) {
  constexpr int kAhead = 8;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  const int parts = p.top_k * p.splits;  // slot by slot, its splits in order
  for (int first = 0; first < parts; first += kAhead) {
    float4 v[kAhead];
    float w[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      w[i] = 0.f;
      const int s = p.splits == 1 ? first + i : (first + i) / p.splits;
      const int split = p.splits == 1 ? 0 : (first + i) % p.splits;
      const int64_t pair = t * p.top_k + s;
      if (first + i < parts && p.ids[pair] >= 0) {
        v[i] = __ldcg(reinterpret_cast<const float4*>(
            p.partial + (static_cast<int64_t>(split) * p.pairs + pair) * p.dim + col));
        w[i] = p.weights[pair];
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      sum.x = fmaf(w[i], v[i].x, sum.x);
      sum.y = fmaf(w[i], v[i].y, sum.y);
      sum.z = fmaf(w[i], v[i].z, sum.z);
      sum.w = fmaf(w[i], v[i].w, sum.w);
    }
  }
  if (p.y_f32)
    *reinterpret_cast<float4*>(static_cast<float*>(p.y) + t * p.y_stride + col) = sum;
  else
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.y) + t * p.y_stride + col) =
        make_uint2(pack2(sum.x, sum.y), pack2(sum.z, sum.w));
}

// Pairs: maps of the scales' tiles (rows of 512 bytes), which tiled loads take so that they can
// report to the other CTA's barrier; the other variants' plain bulk copies need none.
struct ScaleMaps {
  CUtensorMap a, b0, b1;
};
struct NoScaleMaps {};
template <int kVariant>
using ScaleMapsOf = std::conditional_t<kVariant == kPairs, ScaleMaps, NoScaleMaps>;

template <bool kMx, int kVariant, int kPhase>
__global__ void __launch_bounds__(Shape<kVariant>::kThreads, Shape<kVariant>::kCtasPerSm)
    product(const __grid_constant__ ExpertsParams p, const __grid_constant__ CUtensorMap map_a,
            const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_b1,
            const __grid_constant__ ScaleMapsOf<kVariant> scale_maps) {
  using S = Shape<kVariant>;
  constexpr bool kPair = S::kPair;
  constexpr int kCtas = S::kCtas, kStages = S::kStages;
  constexpr uint32_t kStageBytes = S::kStageBytes;
  constexpr int kM = kTileM * kCtas, kN = kTileB * kCtas;  // of one MMA
  constexpr int kElems = kMx ? 128 : 64;    // elements of K per stage
  constexpr int kStepElems = kMx ? 32 : 16; // per MMA (32 bytes)
  // weight rows of a tile from one matrix: phase 1 takes half of them from w1, half from w3
  constexpr int kCols = kPhase == 1 ? kN / 2 : kN;
  constexpr bool kGather = kPhase == 1 && !kPair;  // the A rows come from the gather warps
  constexpr int kBoxA = S::kBoxA;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* s_scale = base + kStages * kStageBytes;  // per stage: A scales, then B scales
  Ctl& ctl = *reinterpret_cast<Ctl*>(s_scale + kStages * kScaleBytes);
  int32_t* first_unit = kPair ? reinterpret_cast<int32_t*>(&ctl + 1) : ctl.first_tile;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = kPair ? static_cast<int>(cluster_ctarank()) : 0;
  const int64_t first = blockIdx.x / kCtas, step = gridDim.x / kCtas;
  const long long limit = p.wait_cycles > 0 ? p.wait_cycles : kWaitCycles;
  // rank 0's copy of a barrier (the one the issuer waits on)
  const auto lead = [](uint64_t* bar) { return map_shared_rank(smem_u32(bar), 0); };

  if (warp == S::kIssueWarp) {
    if constexpr (kPair) {
      tmem_alloc_pair<S::kTmem>(&ctl.tmem_base);
      tmem_relinquish_pair();
    } else {
      tmem_alloc<S::kTmem>(&ctl.tmem_base);
      tmem_relinquish();
    }
  }
  if (warp == S::kProducerWarp && lane == 0) {
    for (int b = 0; b < kStages; ++b) {
      // the producer, the gather warps, and in rank 0 of a pair rank 1's producer
      mbar_init(&ctl.full[b], 1 + (kGather ? S::kGatherWarps : 0) + (kPair && rank == 0 ? 1 : 0));
      mbar_init(&ctl.empty[b], 1);
    }
    mbar_init(&ctl.acc_full, 1);
    mbar_init(&ctl.acc_free, S::kEpilogueWarps * kCtas);
    mbar_init(&ctl.drained, 1);
    ctl.abort = 0;
    fence_barrier_init();
    if (!kGather) tma_prefetch_desc(&map_a);
    tma_prefetch_desc(&map_b0);
    if (kPhase == 1) tma_prefetch_desc(&map_b1);
  }
  // The call's first launch waits for what is before it on the stream, and only then lets the
  // next one start: that one may read the plan and the weights at once.
  if (kGather) grid_dep_wait();
  grid_dep_launch();
  if (kVariant == kFew && kPhase == 1 && blockIdx.x == 0)
    for (int i = threadIdx.x; i < (p.dim + kTileB - 1) / kTileB; i += S::kThreads) p.arrived[i] = 0;
  read_plan<kCtas, S::kRowsA>(p, ctl.first_row, ctl.first_tile, first_unit);
  tc_fence_before();
  if constexpr (kPair) cluster_sync();  // both CTAs' barriers exist, TMEM is allocated
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem_base;
  volatile int32_t* abort_flag = &ctl.abort;
  // the same shared memory of the pair's other CTA (which stays until the teardown's cluster_sync)
  const auto peer = [&](const void* at) { return map_shared_rank(smem_u32(at), rank ^ 1); };
  const auto report_timeout = [&]() {
    if (p.status) atomicOr(p.status, DARD_STATUS_TIMEOUT);
  };
  const auto give_up = [&]() {
    *abort_flag = 1;
    if constexpr (kPair) store_cluster(peer(&ctl.abort), 1);
    report_timeout();
  };
  const int split_stages = kPhase == 2 ? p.split_stages : p.k_stages;
  const auto wait = [&](uint64_t* bar, uint32_t parity) {
    return try_wait<kPair>(bar, parity) || wait_slow<kPair>(bar, parity, limit, abort_flag);
  };
  // the same by every lane of a warp, with one verdict
  const auto warp_wait = [&](uint64_t* bar, uint32_t parity) {
    return __all_sync(0xffffffffu, wait(bar, parity)) != 0;
  };

  if (warp == S::kProducerWarp) {
    // -------------------------------------------------------------- TMA producer
    // As the issuer: uniform over the warp, one elected lane issues. (Copies issued by several
    // lanes, or by a lane of a diverged warp, cost the warp about 80 cycles each.)
    int e = 0, use = 0;
    bool ok = true;
    Tile t;
    const bool issue = elect_one();
    bool waited = kGather;  // for the launch before this one, which writes the rows of A
    Ring ring;
    for (int64_t w = first; ok && get_tile<kVariant>(p, ctl, first_unit, rank, w, e, t); w += step) {
      const int boxes_a = kGather ? 0 : (max(t.count, 0) + kBoxA - 1) / kBoxA;
      const int k0 = t.split * split_stages, k1 = min(p.k_stages, k0 + split_stages);
      const int n0 = t.n * kCols;
      // tiles of weight scales: phase 1 one of w1 and one of w3; phase 2 one per 128 columns
      const bool second = kPhase == 1 || (kN > 128 && n0 + 128 < p.n_elems);
      uint32_t bytes = kBytesB + boxes_a * kBoxA * kStageK;
      if (kMx) bytes += (second ? 2 : 1) * kMxTileBytes + (boxes_a > 0 ? kMxTileBytes : 0);
      // first tiles of scales of this tile's rows: k_stages of them side by side
      const int64_t at_b = (static_cast<int64_t>(t.e) * ((p.n_elems + 127) / 128) + n0 / 128) * p.k_stages;
      const int64_t at_b1 = kPhase == 1 ? at_b : at_b + p.k_stages;
      const int64_t at_a = static_cast<int64_t>(t.row_tile) * p.k_stages;
      // A pair's CTA without rows: zeros (a box outside the map) into each stage, once a tile.
      // Power bounds long runs of the largest calls (the clock falls from 2070 to 1600-1900 MHz),
      // and zeros take less of it than another tile's rows: 800 rows of 4096 x 12288, call after
      // call, 115.0 us against 116.8.
      const auto no_rows = [&](int k) { return kPair && boxes_a == 0 && k - k0 < kStages; };
      const auto load_b = [&](int k, int b) {
        uint8_t* sb = base + b * kStageBytes + S::kBytesA;
        uint8_t* ss = s_scale + b * kScaleBytes;
        const uint32_t all = bytes + (no_rows(k) ? kBoxA * kStageK : 0);
        if constexpr (kPair) {
          const uint32_t bar = lead(&ctl.full[b]);
          arrive_expect_tx_cluster(bar, all);
          if (use != p.test_drop) {
            if constexpr (kPhase == 1)
              tma_load_3d_pair(sb, rank == 1 ? &map_b1 : &map_b0, bar, k * kElems, n0, t.e);
            else
              tma_load_3d_pair(sb, &map_b0, bar, k * kElems, n0 + rank * kTileB, t.e);
          }
          if constexpr (kMx) {
            tma_load_2d_pair(ss + kMxTileBytes, &scale_maps.b0, bar, 0, static_cast<int32_t>(at_b + k));
            if (second)
              tma_load_2d_pair(ss + 2 * kMxTileBytes, &scale_maps.b1, bar, 0, static_cast<int32_t>(at_b1 + k));
          }
        } else {
          uint64_t* bar = &ctl.full[b];
          mbar_arrive_expect_tx(bar, all);
          if (use != p.test_drop) {
            tma_load_3d(sb, &map_b0, bar, k * kElems, n0, t.e);
            if constexpr (kPhase == 1)  // 64 rows of each matrix
              tma_load_3d(sb + 64 * kStageK, &map_b1, bar, k * kElems, n0, t.e);
          }
          if constexpr (kMx) {
            bulk_load(ss + kMxTileBytes, p.scale_b[0] + (at_b + k) * kMxTileBytes, kMxTileBytes, bar);
            if constexpr (kPhase == 1)
              bulk_load(ss + 2 * kMxTileBytes, p.scale_b[1] + (at_b + k) * kMxTileBytes, kMxTileBytes, bar);
          }
        }
      };
      const auto load_a = [&](int k, int b) {
        uint8_t* sa = base + b * kStageBytes;
        uint8_t* ss = s_scale + b * kScaleBytes;
        if constexpr (kPair) {
          const uint32_t bar = lead(&ctl.full[b]);
          if (boxes_a > 0 || no_rows(k))
            tma_load_2d_pair(sa, &map_a, bar, k * kElems,
                             (boxes_a > 0 ? t.row_tile : p.max_row_tiles) * kTileM);
          if (kMx && boxes_a > 0)
            tma_load_2d_pair(ss, &scale_maps.a, bar, 0, static_cast<int32_t>(at_a + k));
        } else {
          uint64_t* bar = &ctl.full[b];
          for (int i = 0; i < boxes_a; ++i)
            tma_load_2d(sa + i * kBoxA * kStageK, &map_a, bar, k * kElems,
                        t.row_tile * kTileM + i * kBoxA);
          if (kMx && boxes_a > 0)
            bulk_load(ss, p.a_scale + (at_a + k) * kMxTileBytes, kMxTileBytes, bar);
        }
      };
      int k = k0;
      if (!waited) {
        // the first stages' weights are on their way while the launch before this one finishes
        const int ahead = min(k1 - k0, kStages);
        if (issue) {
          for (int i = 0; i < ahead; ++i, ++use) load_b(k0 + i, i);
          use = 0;
        }
        grid_dep_wait();
        waited = true;
        if (issue)
          for (int i = 0; i < ahead; ++i) load_a(k0 + i, i);
        __syncwarp();
        use = ahead;
        k += ahead;
        for (int i = 0; i < ahead; ++i) ring.next<kStages>();
      }
      for (; k < k1; ++k, ++use) {
        ok = warp_wait(&ctl.empty[ring.b], ring.phase ^ 1);
        if (!ok) break;
        if (issue) {
          load_b(k, ring.b);
          load_a(k, ring.b);
        }
        __syncwarp();
        ring.next<kStages>();
      }
    }
    // Without a tile too: a launch ends after the one before it, which otherwise could still read
    // the plan or write x's copy when the call seems over to what follows it.
    if (!waited) grid_dep_wait();
    if (!ok && lane == 0) give_up();
    if constexpr (kPair) {  // (the teardown waits for copies in flight)
      if (lane == 0) {
        ctl.uses[rank] = use;
        store_cluster(peer(&ctl.uses[rank]), use);
      }
    } else if (!ok) {
      // copies in flight land before shared memory is released: the last use of each stage
      for (int u = max(0, use - kStages); u < use; ++u)
        mbar_wait(&ctl.full[u % kStages], (u / kStages) & 1, limit);
    }
    __syncwarp();
  } else if (warp == S::kIssueWarp) {
    if (rank == 0) {
      // ------------------------------------------------------------ MMA issuer
      // The whole warp walks the loop, so that what it computes is uniform over the warp; one
      // elected lane issues.
      int e = 0, tiles = 0;
      bool ok = true;
      Tile t;
      Ring ring;
      const bool issue = elect_one();
      const uint64_t desc_a = smem_desc_sw128(smem_u32(base), 16, 1024);
      const uint64_t desc_s = scale_desc(smem_u32(s_scale));
      uint32_t sfa = tmem + S::kScaleCol;  // scales of two stages, 16 columns apart
      bool ready = false;                  // the stage at `ring` is known to be full
      for (int64_t w = first; ok && get_tile<kVariant>(p, ctl, first_unit, rank, w, e, t); w += step, ++tiles) {
        ok = tiles == 0 || warp_wait(&ctl.acc_free, (tiles - 1) & 1);
        if (!ok) break;
        tc_fence_after();
        const int k0 = t.split * split_stages, k1 = min(p.k_stages, k0 + split_stages);
        // 64 weight rows of a matrix are half of a tile of 128 scales
        const uint32_t half = kPhase == 1 && kCols == 64 ? (t.n & 1) * 2 : 0;
        for (int k = k0; k < k1; ++k) {
          // (a wait, even one that is over, costs some 120 cycles, a fifth of a stage: the next
          // stage's barrier is looked at while this one's MMAs are issued)
          if (!ready) ok = warp_wait(&ctl.full[ring.b], ring.phase);
          if (!ok) break;
          tc_fence_after();
          Ring next = ring;
          next.next<kStages>();
          const bool look = mbar_test<kPair>(&ctl.full[next.b], next.phase);
          if (issue) {
            // descriptors count 16-byte units
            const uint64_t da = desc_a + ring.b * (kStageBytes / 16), db = da + S::kBytesA / 16;
            const uint32_t sfb = sfa + 8;
            if constexpr (kMx) {
              const uint64_t ds = desc_s + ring.b * (kScaleBytes / 16);
              copy_scales<kPair>(sfa, ds);
              copy_scales<kPair>(sfb, ds + kMxTileBytes / 16);
              if (kPhase == 1 || kN > 128) copy_scales<kPair>(sfb + 4, ds + 2 * kMxTileBytes / 16);
            }
            const int left = p.k_elems - k * kElems;  // the last stage may hold fewer steps
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
              if (ks * kStepElems >= left) break;
              const uint32_t acc = (k > k0 || ks > 0) ? 1u : 0u;
              const uint64_t off = ks * 32 / 16;
              if constexpr (!kMx && kPair) {
                mma_ss_pair(tmem, da + off, db + off, idesc_bf16_f32(kM, kN, 0, 0), acc);
              } else if constexpr (!kMx) {
                mma_ss(tmem, da + off, db + off, idesc_bf16_f32(kM, kN, 0, 0), acc);
              } else if constexpr (kPhase == 1 && kCols == 64) {
                // w1's and w3's scales lie in different tiles: one MMA for each
                mma_mx<kPair>(tmem, da + off, db + off, idesc_mx(kM, 64, ks), sfa, sfb + half, acc);
                mma_mx<kPair>(tmem + 64, da + off, db + off + 64 * kStageK / 16, idesc_mx(kM, 64, ks),
                              sfa, sfb + 4 + half, acc);
              } else {
                mma_mx<kPair>(tmem, da + off, db + off, idesc_mx(kM, kN, ks), sfa, sfb, acc);
              }
            }
            if constexpr (kPair) mma_commit_pair(&ctl.empty[ring.b], kBothCtas);
            else mma_commit(&ctl.empty[ring.b]);
            if (k == k1 - 1) {
              if constexpr (kPair) mma_commit_pair(&ctl.acc_full, kBothCtas);
              else mma_commit(&ctl.acc_full);
            }
          }
          ready = __all_sync(0xffffffffu, look);
          ring = next;
          sfa ^= 16;
        }
      }
      if (!ok && lane == 0) give_up();
      if (issue) {
        if constexpr (kPair) mma_commit_pair(&ctl.drained, kBothCtas);
        else mma_commit(&ctl.drained);
      }
    }
    __syncwarp();
  } else if (warp >= S::kGatherWarp) {
    // -------------------------------------------------------------- rows of x, by token
    if (kGather) {
      const int g = warp - S::kGatherWarp;
      constexpr int kRows = S::kRowsA / S::kGatherWarps;  // of this warp: g * kRows ..
      constexpr int kCopies = kRows / 4;            // a warp copies four rows (8 lanes each) at once
      const int chunk = lane & 7, sub = lane >> 3;
      const char* xb = static_cast<const char*>(p.x) + chunk * 16;
      const int row_bytes = p.k_elems * (kMx ? 1 : 2);
      int e = 0, pending = 0;
      bool ok = true;
      Tile t;
      Ring ring, oldest;  // the next stage; the first of the `pending` that are not announced
      // tells the issuer of the oldest stages, all but `left`, whose copies have landed
      const auto announce = [&](int left) {
        fence_proxy_async_smem();  // before the tensor core reads what was written here
        __syncwarp();
        for (; pending > left; --pending) {
          if (lane == 0) mbar_arrive(&ctl.full[oldest.b]);
          oldest.next<kStages>();
        }
      };
      for (int64_t w = first; ok && get_tile<kVariant>(p, ctl, first_unit, rank, w, e, t); w += step) {
        int64_t from[kCopies];  // byte offset of the token's row; -1: no row
        const uint4* src[2] = {nullptr, nullptr};  // scales of rows g * kRows + lane (+ 32)
#pragma unroll
        for (int h = 0; h < kRows / 32; ++h) {
          const int at = g * kRows + 32 * h + lane;
          const int pair = at < t.count ? __ldg(p.rows + t.row + at) : -1;
          const int token = pair >= 0 && pair < p.pairs ? pair / p.top_k : -1;
          if (kMx && token >= 0)
            src[h] = reinterpret_cast<const uint4*>(p.x_scale + static_cast<int64_t>(token) * p.x_scale_stride);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const int tok = __shfl_sync(0xffffffffu, token, 4 * c + sub);
            from[8 * h + c] = tok >= 0 ? static_cast<int64_t>(tok) * p.x_stride_bytes : -1;
          }
        }
        uint32_t now[2][4] = {}, ahead[2][4] = {};  // [row][stage within a group of four]
        const auto fetch = [&](int group) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (src[h] != nullptr && 4 * group < p.k_stages) v = __ldg(src[h] + group);
            ahead[h][0] = v.x;
            ahead[h][1] = v.y;
            ahead[h][2] = v.z;
            ahead[h][3] = v.w;
          }
        };
        if (kMx) fetch(0);
        for (int k = 0; ok && k < p.k_stages; k += 4) {
          if (kMx) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
              for (int j = 0; j < 4; ++j) now[h][j] = ahead[h][j];
            }
            fetch(k / 4 + 1);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (k + j >= p.k_stages) break;
            const int b = ring.b;
            if (!__all_sync(0xffffffffu, mbar_test<kPair>(&ctl.empty[b], ring.phase ^ 1))) {
              cp_async_wait_all();  // nothing else to do: tell of every stage so far
              announce(0);
            }
            ok = warp_wait(&ctl.empty[b], ring.phase ^ 1);
            if (!ok) break;
            uint8_t* sa = base + b * kStageBytes;
            const int col = (k + j) * kStageK;
            if (col + chunk * 16 < row_bytes) {
#pragma unroll
              for (int c = 0; c < kCopies; ++c) {
                const int row = g * kRows + 4 * c + sub;
                if (from[c] >= 0)
                  cp_async16(sa + row * kStageK + ((chunk ^ (row & 7)) << 4), xb + from[c] + col, 16);
              }
            }
            cp_async_commit();
            if (kMx) {
              uint8_t* ss = s_scale + b * kScaleBytes + lane * 16 + g * (kRows / 32) * 4;
              if constexpr (kRows > 32) *reinterpret_cast<uint2*>(ss) = make_uint2(now[0][j], now[1][j]);
              else *reinterpret_cast<uint32_t*>(ss) = now[0][j];
            }
            ring.next<kStages>();
            if (++pending > kGatherLag) {
              cp_async_wait_group<kGatherLag>();
              announce(kGatherLag);
            }
          }
        }
        cp_async_wait_all();
        announce(0);
      }
      if (!ok && lane == 0) give_up();
      __syncwarp();
    }
  } else {
    // -------------------------------------------------------------- epilogue
    const int quarter = warp & 3;
    const int r = quarter * 32 + lane;  // TMEM lane = row of the tile
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    // 32-column loads of half a tile: a pair's warp takes one half, a single CTA's both in turn
    constexpr int kChunks = kN / 2 / 32;
    int e = 0, tiles = 0;
    bool ok = true;
    Tile t;
    if (kPhase == 2) {
      grid_dep_wait();
      if (p.direct) {
        // tokens without an expert: no pair of theirs reaches any tile
        constexpr int kRun = 32 * S::kEpilogueWarps;
        for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRun + warp * 32; t0 < p.tokens;
             t0 += static_cast<int64_t>(gridDim.x) * kRun) {
          uint32_t missing = __ballot_sync(0xffffffffu, t0 + lane < p.tokens && p.ids[t0 + lane] < 0);
          for (; missing != 0; missing &= missing - 1) {
            const int64_t at = (t0 + __ffs(missing) - 1) * p.y_stride;
            for (int i = lane; i < p.dim; i += 32) {
              if (p.y_f32) static_cast<float*>(p.y)[at + i] = 0.f;
              else static_cast<__nv_bfloat16*>(p.y)[at + i] = __float2bfloat16_rn(0.f);
            }
          }
        }
      }
    }
    for (int64_t w = first; ok && get_tile<kVariant>(p, ctl, first_unit, rank, w, e, t); w += step, ++tiles) {
      const bool in = r < t.count;
      int pair = 0;
      if (kPhase == 2) pair = in ? __ldg(p.rows + t.row + r) : -1;
      ok = wait(&ctl.acc_full, tiles & 1);
      if constexpr (kVariant == kFew && kPhase == 2) ok = epilogue_and<S::kEpilogueWarps>(ok);
      else ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const int half0 = kPair ? warp >> 2 : 0, half1 = kPair ? half0 + 1 : 2;
#pragma unroll 1
      for (int half = half0; half < half1; ++half) {
        uint32_t acc[kChunks][32];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          // phase 1: chunk c < kChunks / 2 of the gate, then the same columns of the value
          const int col = kPhase == 1 ? (c < kChunks / 2 ? 0 : kCols) + half * (kCols / 2) +
                                            32 * (c % (kChunks / 2))
                                      : half * (kN / 2) + 32 * c;
          tmem_ld32(tmem + lanes + col, acc[c]);
        }
        tmem_wait_ld();
        if (half == half1 - 1) {  // the accumulator is in registers: the next tile's MMAs may start
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (kPair) arrive_cluster(lead(&ctl.acc_free));
            else mbar_arrive(&ctl.acc_free);
          }
        }
        // (the arithmetic that follows may not move ahead of that)
#pragma unroll
        for (int c = 0; c < kChunks; ++c) pin32(acc[c]);
        if constexpr (kPhase == 1) {
#pragma unroll
          for (int c = 0; c < kChunks / 2; ++c) {
            const int col = t.n * kCols + half * (kCols / 2) + 32 * c;  // hidden element
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i)
              v[i] = silu(__uint_as_float(acc[c][i])) * __uint_as_float(acc[c + kChunks / 2][i]);
            const int64_t row = static_cast<int64_t>(t.row_tile) * kTileM + r;
            if constexpr (kMx) {
              float m = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) m = max_nan(m, fabsf(v[i]));
              const uint32_t b = mx_scale_byte(m);
              const float s = mx_inverse(b);
              if (in && col < p.hidden) {
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  q[i] = e4m3x4(v[4 * i] * s, v[4 * i + 1] * s, v[4 * i + 2] * s, v[4 * i + 3] * s);
                store32(p.h + row * p.hidden + col, q);
                const int tiles_h = (p.hidden + 127) / 128;
                p.h_scale[(static_cast<int64_t>(t.row_tile) * tiles_h + col / 128) * kMxTileBytes +
                          mx_tile_byte(r, col / 32)] = static_cast<uint8_t>(b);
              }
            } else if (in && col < p.hidden) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                uint32_t q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = pack2(v[16 * i + 2 * j], v[16 * i + 2 * j + 1]);
                store32(p.h + (row * p.hidden + col) * 2 + 32 * i, q);
              }
            }
          }
        } else {
          const bool store = pair >= 0 && pair < p.pairs;
          const float weight = p.direct && store ? p.weights[pair] : 1.f;
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const int col = t.n * kN + half * (kN / 2) + 32 * c;
            if (!store || col >= p.dim) continue;
            const uint32_t (&a)[32] = acc[c];
            if (!p.direct) {
              float* to = p.partial + (static_cast<int64_t>(t.split) * p.pairs + pair) * p.dim + col;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = a[8 * i + j];
                store32(to + 8 * i, q);
              }
            } else if (!p.y_f32) {
              uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.y) +
                                                    pair * p.y_stride + col);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t q[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  q[j] = pack2(__uint_as_float(a[8 * i + 2 * j]) * weight,
                               __uint_as_float(a[8 * i + 2 * j + 1]) * weight);
                dst[i] = make_uint4(q[0], q[1], q[2], q[3]);
              }
            } else {
              float4* dst = reinterpret_cast<float4*>(static_cast<float*>(p.y) + pair * p.y_stride + col);
#pragma unroll
              for (int i = 0; i < 8; ++i)
                dst[i] = make_float4(__uint_as_float(a[4 * i]) * weight, __uint_as_float(a[4 * i + 1]) * weight,
                                     __uint_as_float(a[4 * i + 2]) * weight,
                                     __uint_as_float(a[4 * i + 3]) * weight);
            }
          }
        }
      }
      if constexpr (kVariant == kFew && kPhase == 2) {
        // The last of a column tile's tiles adds them up (in slot order, whichever is last).
        if (!p.direct) {
          __threadfence();
          epilogue_and<S::kEpilogueWarps>(true);
          if (threadIdx.x == 0) {
            const int all = ctl.first_tile[p.experts] * p.splits;
            ctl.last = atomicAdd(p.arrived + t.n, 1) == all - 1;
          }
          epilogue_and<S::kEpilogueWarps>(true);
          if (ctl.last) {
            __threadfence();
            for (int i = threadIdx.x; i < p.tokens * 32; i += 32 * S::kEpilogueWarps) {
              const int col = t.n * kN + 4 * (i % 32);
              if (col < p.dim) combine_columns(p, i / 32, col);
            }
          }
        }
      }
    }
    if (kVariant == kFew && kPhase == 2 && !p.direct && ctl.first_tile[p.experts] == 0) {
      // no token has an expert, and no tile says so
      for (int64_t i = static_cast<int64_t>(blockIdx.x) * 128 + threadIdx.x;
           i < static_cast<int64_t>(p.tokens) * (p.dim / 4); i += static_cast<int64_t>(gridDim.x) * 128)
        combine_columns(p, static_cast<int>(i / (p.dim / 4)), 4 * static_cast<int>(i % (p.dim / 4)));
    }
    if (!ok && lane == 0) give_up();
    __syncwarp();
  }
  // ---------------------------------------------------------------- teardown
  tc_fence_before();
  if constexpr (kPair) {
    cluster_sync();  // no CTA leaves while the other may signal its barriers
    if (ctl.abort != 0) {
      // Both CTAs are here. Copies in flight land before shared memory is released: rank 0's
      // barriers tell, once the rank that has filled fewer stages (by at most kStages: no stage is
      // filled again before both ranks' part of it was used) has arrived for the others.
      if (rank == 0 && warp == S::kProducerWarp) {
        const int low = min(ctl.uses[0], ctl.uses[1]), high = max(ctl.uses[0], ctl.uses[1]);
        if (lane == 0)
          for (int u = low; u < high; ++u) mbar_arrive(&ctl.full[u % kStages]);
        __syncwarp();
        for (int u = max(0, high - kStages); u < high; ++u)
          mbar_wait(&ctl.full[u % kStages], (u / kStages) & 1, limit);
        __syncwarp();
      }
      cluster_sync();
    }
  } else {
    __syncthreads();
  }
  if (warp == S::kIssueWarp) {
    if (!mbar_wait(&ctl.drained, 0, limit) && lane == 0) report_timeout();
    __syncwarp();
    tc_fence_after();
    if constexpr (kPair) tmem_dealloc_pair<S::kTmem>(tmem);
    else tmem_dealloc<S::kTmem>(tmem);
  }
}

// x (and its scales) in the plan's order, every expert's rows from a row tile's start: one or
// a few warps per pair of the plan. The first pair's row is on its way while the plan is read.
template <bool kMx>
__global__ void __launch_bounds__(256) gather_rows(const __grid_constant__ ExpertsParams p) {
  grid_dep_wait();  // the call's first launch (see product)
  grid_dep_launch();
  __shared__ int32_t first_row[DARD_MAX_EXPERTS + 1], first_tile[DARD_MAX_EXPERTS + 1],
      first_unit[DARD_MAX_EXPERTS + 1];
  const int lane = threadIdx.x & 31;
  const int64_t row_bytes = static_cast<int64_t>(p.dim) * (kMx ? 1 : 2);
  const int n = static_cast<int>(row_bytes / 16), scale_tiles = (p.dim + 127) / 128;
  const auto token_of = [&](int i) {
    const int pair = i < p.pairs ? p.rows[i] : -1;
    return pair >= 0 && pair < p.pairs ? static_cast<int64_t>(pair / p.top_k) : -1;
  };
  uint4 v[4];
  const auto load = [&](int64_t token, int c) {
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(p.x) + token * p.x_stride_bytes);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + 32 * j < n) v[j] = load16_here(src + c + 32 * j);
  };
  const int warp = blockIdx.x * 8 + (threadIdx.x >> 5), parts = 1 << p.gather_shift;
  int i = warp >> p.gather_shift;
  const int part = warp & (parts - 1), c0 = 128 * part + lane;  // this warp's 16 bytes: c0, c0 + 32, ..
  int64_t token = token_of(i);
  if (token >= 0) load(token, c0);
  read_plan<1, kTileM>(p, first_row, first_tile, first_unit);
  __syncthreads();
  while (i < p.pairs) {
    int lo = 0, hi = p.experts;  // first_row[lo] <= i < first_row[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first_row[mid] <= i) lo = mid;
      else hi = mid;
    }
    const int at = i - first_row[lo], tile = first_tile[lo] + at / kTileM;
    if (token >= 0 && at >= 0 && i < first_row[lo + 1] && tile < first_tile[lo + 1]) {
      const int64_t row = static_cast<int64_t>(tile) * kTileM + at % kTileM;
      uint4* dst = reinterpret_cast<uint4*>(p.xg + row * row_bytes);
      for (int c = c0; c < n; c += 128 * parts) {
        if (c != c0) load(token, c);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + 32 * j < n) dst[c + 32 * j] = v[j];
      }
      if (kMx && part == 0) {
        const uint32_t* sc = reinterpret_cast<const uint32_t*>(p.x_scale + token * p.x_scale_stride);
        for (int c = lane; c < scale_tiles; c += 32)
          *reinterpret_cast<uint32_t*>(p.xg_scale + (static_cast<int64_t>(tile) * scale_tiles + c) * kMxTileBytes +
                                       mx_tile_byte(at % kTileM, 0)) = __ldg(sc + c);
      }
    }
    i += gridDim.x * 8 >> p.gather_shift;
    token = token_of(i);
    if (token >= 0) load(token, c0);
  }
}

// One thread per four columns of a token. Bound by HBM's reads of what phase 2 has just written:
// 8192 x 8 rows of 4096 fp32 (1.07 GB) 250 us, 4.5 TB/s; cold, 4096 x 4 rows (0.27 GB) 5.7 TB/s.
__global__ void __launch_bounds__(128) combine(const __grid_constant__ ExpertsParams p) {
  grid_dep_launch();
  // (written before the call: here while phase 2 still runs; 1111 tokens x 6 of 40: 87.3 us, 87.8)
  if (static_cast<int>(threadIdx.x) < p.top_k) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * p.top_k + threadIdx.x;
    asm volatile("prefetch.global.L1 [%0];" ::"l"(p.ids + at));
    asm volatile("prefetch.global.L1 [%0];" ::"l"(p.weights + at));
  }
  grid_dep_wait();
  const int col = 4 * (blockIdx.y * 128 + threadIdx.x);
  if (col < p.dim) combine_columns(p, blockIdx.x, col);
}

// ---------------------------------------------------------------- host side
// Rank-2 (planes 0) or rank-3 map of row-major bytes / bf16 with 128-byte swizzle.
bool encode(CUtensorMap* m, const void* ptr, bool mx, uint64_t cols, uint64_t rows, uint64_t planes,
            uint64_t row_bytes, uint32_t box_rows) {
  const auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cols, rows, planes};
  const cuuint64_t strides[2] = {row_bytes, row_bytes * rows};
  const cuuint32_t box[3] = {mx ? 128u : 64u, box_rows, 1};
  const cuuint32_t unit[3] = {1, 1, 1};
  return fn(m, mx ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
            planes ? 3 : 2, const_cast<void*>(ptr), dims, strides, box, unit,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Map of tiles of scales, each a row of 128 words.
bool encode_scales(CUtensorMap* m, const void* ptr, int64_t tiles) {
  const auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {kMxTileBytes / 4, static_cast<cuuint64_t>(tiles)};
  const cuuint64_t strides[1] = {kMxTileBytes};
  const cuuint32_t box[2] = {kMxTileBytes / 4, 1}, unit[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(ptr), dims, strides, box, unit,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A launch that may begin (up to its griddepcontrol.wait) while the one before it on the stream
// still runs, with clusters of `cluster` CTAs. Not copyable: cfg points at attr.
struct Launch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  Launch(dim3 grid, unsigned block, size_t smem, cudaStream_t stream, unsigned cluster = 1) {
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
  }
  Launch(const Launch&) = delete;
  Launch& operator=(const Launch&) = delete;
};

// Clusters of two CTAs of this kernel that fit on the device at once, looked up once per device.
template <class F>
int max_pairs(F* kernel, std::atomic<int>* cache) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return sm_count() / 2;
  int n = cache[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  const Launch l(dim3(2 * 64), Shape<kPairs>::kThreads, smem_bytes<kPairs>(), nullptr, 2);
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &l.cfg) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    return sm_count() / 2;
  }
  cache[dev].store(n, std::memory_order_relaxed);
  return n;
}

// The maps of one phase's launch: rows of A, weights, and (pairs, MXFP8) their scales.
struct Maps {
  CUtensorMap a, b0, b1;
  ScaleMaps scales;
};

template <bool kMx, int kVariant, int kPhase>
cudaError_t launch_product(const ExpertsParams& p, int64_t tiles, const Maps& m, cudaStream_t stream) {
  using S = Shape<kVariant>;
  static std::atomic<uint64_t> done{0};
  static std::atomic<int> pairs[64];
  const auto kernel = product<kMx, kVariant, kPhase>;
  const cudaError_t e = ensure_smem_attr(kernel, smem_bytes<kVariant>(), done);
  if (e != cudaSuccess) return e;
  const int64_t most = S::kPair ? max_pairs(kernel, pairs) : sm_count() * S::kCtasPerSm;
  const unsigned ctas = static_cast<unsigned>(std::min<int64_t>(tiles, most)) * S::kCtas;
  const Launch l(dim3(ctas), S::kThreads, smem_bytes<kVariant>(), stream, S::kCtas);
  if constexpr (S::kPair) return cudaLaunchKernelEx(&l.cfg, kernel, p, m.a, m.b0, m.b1, m.scales);
  else return cudaLaunchKernelEx(&l.cfg, kernel, p, m.a, m.b0, m.b1, NoScaleMaps{});
}

template <bool kMx, int kPhase>
cudaError_t launch_phase(const ExpertsParams& p, int variant, int64_t tiles, const Maps& m,
                         cudaStream_t s) {
  return variant == kPairs    ? launch_product<kMx, kPairs, kPhase>(p, tiles, m, s)
         : variant == kSingle ? launch_product<kMx, kSingle, kPhase>(p, tiles, m, s)
                              : launch_product<kMx, kFew, kPhase>(p, tiles, m, s);
}

constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Sizes that follow from a call's sizes alone.
struct Plan {
  int64_t pairs, row_tiles;  // at most so many row tiles, whatever the plan
  int variant1, variant2;    // of each phase
  int64_t tiles1, tiles2;    // tiles of each phase, at most (few: where a token's experts differ)
  int splits, split_stages;
  size_t arrived_bytes, h_bytes, h_scale_bytes, partial_bytes, xg_bytes, xg_scale_bytes;
  bool direct;  // phase 2 writes y itself
  // x in the plan's order is read for the last time in phase 1, the pairs' products are written
  // in phase 2: they share their bytes
  size_t bytes() const {
    return arrived_bytes + h_bytes + h_scale_bytes + std::max(partial_bytes, xg_bytes + xg_scale_bytes);
  }
};

// Few tokens (few rows per expert): kFew, in both phases (against kSingle, 8 of 64
// experts of 2048 x 1024: 1 token 22.0 / 22.4 us, 8 51 / 62, 32 85 / 87, or 90 / 88 where some experts
// have more rows than others; bf16 26.9 / 32.3, 80 / 94, 140 / 146). Else pairs of CTAs, unless their
// tiles (their count, over the row tiles that the call can have) are fewer than the pairs of SMs,
// or than half of those where the experts have full row tiles on average: then single ones. (800
// rows of one expert, phase 2 of 4096 x 12288, 64 tiles: 109 against 118 us for the call; both phases
// 107 against 150, bf16 186 against 263; 200 rows of 8 experts, 1536 x 768, 48 and 48 tiles: 18.2
// against 16.5 us, bf16 23.4 against 22.1.) Where even single tiles leave
// SMs idle in phase 2 (few rows, a long reduction), the reduction is split, into runs of at least
// four stages (one expert of 4096 x 12288: 1 row 39.4 us, whole 50.8, bf16 59.6, 84.8; 100 rows
// 55.8, whole 72.9, bf16 86, 128).
Plan make_plan(int64_t tokens, int experts, int top_k, int dim, int hidden, bool mx) {
  Plan q = {};
  q.pairs = tokens * top_k;
  const int64_t used = std::min<int64_t>(experts, q.pairs);  // experts with rows, at most
  const int64_t row_tiles = q.pairs / kTileM + used;  // where no tile is of kFew
  const int64_t row_pairs = q.pairs / (2 * kTileM) + used;
  const int64_t sms = sm_count();
  const auto columns = [](int n, int per) { return static_cast<int64_t>((n + per - 1) / per); };
  const bool few = tokens <= kFewTokens;
  q.row_tiles = few ? used + (q.pairs - used) / Shape<kFew>::kRowsA : row_tiles;
  const int64_t enough = q.pairs >= kTileM * used ? sms / 4 : sms / 2;
  q.variant1 = few ? kFew : row_pairs * columns(hidden, 128) >= enough ? kPairs : kSingle;
  q.variant2 = few ? kFew : row_pairs * columns(dim, 256) >= enough ? kPairs : kSingle;
  q.tiles1 = q.variant1 == kPairs ? row_pairs * columns(hidden, 128) : row_tiles * columns(hidden, 64);
  q.tiles2 = q.variant2 == kPairs ? row_pairs * columns(dim, 256) : row_tiles * columns(dim, 128);
  const int stages = (hidden + (mx ? 127 : 63)) / (mx ? 128 : 64);
  int64_t splits = 1;
  if (q.variant2 != kPairs && q.tiles2 * 2 <= sms)
    splits = std::max<int64_t>(1, std::min<int64_t>(sms / q.tiles2, stages / 4));
  q.split_stages = static_cast<int>((stages + splits - 1) / splits);
  q.splits = (stages + q.split_stages - 1) / q.split_stages;
  q.tiles2 *= q.splits;
  const size_t rows = static_cast<size_t>(q.row_tiles) * kTileM;
  q.h_bytes = up256(rows * hidden * (mx ? 1 : 2));
  q.h_scale_bytes = mx ? up256(static_cast<size_t>(q.row_tiles) * ((hidden + 127) / 128) * kMxTileBytes) : 0;
  q.arrived_bytes = few ? up256(static_cast<size_t>(columns(dim, kTileB)) * 4) : 0;
  if (q.variant1 == kPairs) {
    q.xg_bytes = up256(rows * dim * (mx ? 1 : 2));
    q.xg_scale_bytes = mx ? up256(static_cast<size_t>(q.row_tiles) * ((dim + 127) / 128) * kMxTileBytes) : 0;
  }
  q.direct = top_k == 1 && q.splits == 1;
  if (!q.direct)
    q.partial_bytes = up256(static_cast<size_t>(q.splits) * q.pairs * dim * 4);
  return q;
}

bool sizes_ok(int64_t tokens, int64_t experts, int64_t top_k, int64_t dim, int64_t hidden) {
  const auto width = [](int64_t n) { return n >= 32 && n % 32 == 0 && n <= DARD_EXPERTS_MAX_DIM; };
  return tokens >= 0 && experts >= 1 && experts <= DARD_MAX_EXPERTS && top_k >= 1 &&
         top_k <= std::min<int64_t>(experts, DARD_MAX_TOP_K) && tokens * top_k <= (1 << 24) &&
         width(dim) && width(hidden);
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace
}  // namespace dard

using namespace dard;

extern "C" {

size_t dard_experts_workspace_size(int32_t tokens, int32_t experts, int32_t top_k, int32_t dim,
                                   int32_t hidden) {
  if (!sizes_ok(tokens, experts, top_k, dim, hidden) || tokens == 0) return 0;
  // The most that any count up to this one needs. It falls only where fewer tokens have more row
  // tiles (few) or a reduction that is split (at most half as many tiles as SMs, so at most half
  // as many row tiles of 128 pairs): those counts are looked at one by one.
  size_t most = 0;
  const int64_t row_tiles = sm_count() / 2 / ((dim + kTileB - 1) / kTileB);
  const int64_t alone = std::max<int64_t>(kFewTokens, (row_tiles + 1) * kTileM / top_k);
  for (int mx = 0; mx < 2; ++mx) {
    for (int64_t t = 1; t <= std::min<int64_t>(tokens, alone); ++t)
      most = std::max(most, make_plan(t, experts, top_k, dim, hidden, mx != 0).bytes());
    most = std::max(most, make_plan(tokens, experts, top_k, dim, hidden, mx != 0).bytes());
  }
  return most;
}

dard_status dard_experts(const dard_experts_args* a, void* stream) {
  report(DARD_OK, "%s", "");
  if (!a) return report(DARD_ERR_NULL, "args is NULL");
  if (a->dtype != DARD_MXFP8 && a->dtype != DARD_BF16)
    return report(DARD_ERR_VALUE, "dtype %d is neither DARD_MXFP8 nor DARD_BF16", a->dtype);
  if (a->y_dtype != DARD_BF16 && a->y_dtype != DARD_F32)
    return report(DARD_ERR_VALUE, "y_dtype %d is neither DARD_F32 nor DARD_BF16", a->y_dtype);
  if (a->experts < 1 || a->experts > DARD_MAX_EXPERTS)
    return report(DARD_ERR_SHAPE, "experts %d outside 1..%d", a->experts, DARD_MAX_EXPERTS);
  if (a->top_k < 1 || a->top_k > std::min(a->experts, DARD_MAX_TOP_K))
    return report(DARD_ERR_SHAPE, "top_k %d outside 1..min(experts, %d)", a->top_k, DARD_MAX_TOP_K);
  if (!sizes_ok(a->tokens, a->experts, a->top_k, a->dim, a->hidden))
    return report(DARD_ERR_SHAPE,
                  "tokens %d (tokens * top_k in 0..2^24), dim %d, hidden %d (multiples of 32 in "
                  "32..%d)",
                  a->tokens, a->dim, a->hidden, DARD_EXPERTS_MAX_DIM);
  const bool mx = a->dtype == DARD_MXFP8;
  if (a->x_stride < a->dim || a->y_stride < a->dim || (mx && a->x_scale_stride < a->dim / kMxBlock))
    return report(DARD_ERR_SHAPE, "a row stride is below dim (x_scale_stride: dim / 32)");
  if (a->tokens == 0) return DARD_OK;
  if (!a->x || !a->w1 || !a->w3 || !a->w2 || !a->ids || !a->weights || !a->offsets || !a->rows ||
      !a->y)
    return report(DARD_ERR_NULL, "an input or y is NULL");
  if (mx && (!a->x_scale || !a->w1_scale || !a->w3_scale || !a->w2_scale))
    return report(DARD_ERR_NULL, "a scale pointer is NULL with dtype DARD_MXFP8");
  const int esz = mx ? 1 : 2, ysz = a->y_dtype == DARD_BF16 ? 2 : 4;
  if (!aligned(a->x, 16) || !aligned(a->w1, 16) || !aligned(a->w3, 16) || !aligned(a->w2, 16) ||
      !aligned(a->y, 16) || a->x_stride * esz % 16 != 0 || a->y_stride * ysz % 16 != 0)
    return report(DARD_ERR_ALIGN, "x, the weights, y and the row pitches must be multiples of 16 "
                                  "bytes");
  if (mx && (!aligned(a->x_scale, 16) || a->x_scale_stride % 16 != 0 || !aligned(a->w1_scale, 16) ||
             !aligned(a->w3_scale, 16) || !aligned(a->w2_scale, 16)))
    return report(DARD_ERR_ALIGN, "the scales and x_scale_stride must be multiples of 16 bytes");
  const Plan q = make_plan(a->tokens, a->experts, a->top_k, a->dim, a->hidden, mx);
  const size_t need = q.bytes();
  if (!a->workspace || a->workspace_bytes < need)
    return report(DARD_ERR_WORKSPACE, "workspace of %zu bytes needed", need);
  if (!aligned(a->workspace, 256)) return report(DARD_ERR_ALIGN, "workspace must be 256-byte aligned");

  ExpertsParams p = {};
  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  p.offsets = a->offsets;
  p.rows = a->rows;
  p.ids = a->ids;
  p.weights = a->weights;
  p.x = a->x;
  p.x_stride_bytes = a->x_stride * esz;
  p.x_scale = a->x_scale;
  p.scale_b[0] = a->w1_scale;
  p.scale_b[1] = a->w3_scale;
  p.arrived = reinterpret_cast<int32_t*>(ws);
  p.h = ws + q.arrived_bytes;
  p.h_scale = p.h + q.h_bytes;
  p.xg = p.h_scale + q.h_scale_bytes;
  p.partial = reinterpret_cast<float*>(p.xg);
  p.xg_scale = p.xg + q.xg_bytes;
  p.y = a->y;
  p.status = a->status;
  p.x_scale_stride = a->x_scale_stride;
  p.y_stride = a->y_stride;
  p.tokens = a->tokens;
  p.experts = a->experts;
  p.top_k = a->top_k;
  p.dim = a->dim;
  p.hidden = a->hidden;
  p.pairs = static_cast<int32_t>(q.pairs);
  p.max_row_tiles = static_cast<int32_t>(q.row_tiles);
  p.y_f32 = a->y_dtype == DARD_F32;
  p.direct = q.direct;
  p.test_drop = -1;
  // Test hooks (failure-path tests; unset in normal operation): a wait bound, and a stage whose
  // weights never arrive.
  if (const char* w = std::getenv("DARD_TEST_WAIT_CYCLES")) p.wait_cycles = std::atoll(w);
  if (const char* d = std::getenv("DARD_TEST_DROP_KV")) p.test_drop = std::atoi(d);

  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int stage = mx ? 128 : 64;
  cudaError_t e = std::getenv("DARD_TEST_FAIL_LAUNCH") ? cudaErrorLaunchFailure : cudaSuccess;
  Maps m = {};
  // phase 1: rows of x (in the plan's order, or gathered by the kernel itself) and of w1 and w3
  const uint64_t drow = static_cast<uint64_t>(a->dim) * esz, hrow = static_cast<uint64_t>(a->hidden) * esz;
  const uint64_t rows = static_cast<uint64_t>(q.row_tiles) * kTileM;
  const bool pair1 = q.variant1 == kPairs, pair2 = q.variant2 == kPairs;
  const uint32_t box1 = pair1 ? 128 : 64;
  // tiles of scales of all rows of x or h (dtiles, htiles per row tile), and of the weights
  const int64_t dtiles = (a->dim + 127) / 128, htiles = (a->hidden + 127) / 128;
  const int64_t weight_tiles = a->experts * dtiles * htiles;
  if (e == cudaSuccess && (!encode(&m.b0, a->w1, mx, a->dim, a->hidden, a->experts, drow, box1) ||
                           !encode(&m.b1, a->w3, mx, a->dim, a->hidden, a->experts, drow, box1) ||
                           (pair1 && !encode(&m.a, p.xg, mx, a->dim, rows, 0, drow, kTileM)) ||
                           (pair1 && mx && (!encode_scales(&m.scales.a, p.xg_scale, q.row_tiles * dtiles) ||
                                            !encode_scales(&m.scales.b0, a->w1_scale, weight_tiles) ||
                                            !encode_scales(&m.scales.b1, a->w3_scale, weight_tiles)))))
    e = cudaErrorInvalidValue;
  if (!pair1) m.a = m.b0;  // not used
  if (e == cudaSuccess && pair1) {
    // Few pairs: several warps share a row of more than 2 KB, so that it is read in one go (800
    // rows of 4 KB: the call takes 106.4 us, with a warp per row 110.5).
    const int64_t most = 64ll * sm_count();
    while (p.gather_shift < 3 && (2048ull << p.gather_shift) < drow &&
           q.pairs << (p.gather_shift + 1) <= most)
      ++p.gather_shift;
    const int64_t warps = std::min(q.pairs << p.gather_shift, most);
    const Launch l(dim3(static_cast<unsigned>((warps + 7) / 8)), 256, 0, s);
    e = mx ? cudaLaunchKernelEx(&l.cfg, gather_rows<true>, p)
           : cudaLaunchKernelEx(&l.cfg, gather_rows<false>, p);
  }
  if (e == cudaSuccess) {
    p.a_scale = p.xg_scale;
    p.k_elems = a->dim;
    p.n_elems = a->hidden;
    p.n_tiles = (a->hidden + box1 - 1) / box1;
    p.k_stages = (a->dim + stage - 1) / stage;
    p.splits = 1;
    p.split_stages = p.k_stages;
    e = mx ? launch_phase<true, 1>(p, q.variant1, q.tiles1, m, s)
           : launch_phase<false, 1>(p, q.variant1, q.tiles1, m, s);
  }
  // phase 2: rows of h, rows of w2
  if (e == cudaSuccess &&
      (!encode(&m.a, p.h, mx, a->hidden, rows, 0, hrow, pair2 ? Shape<kPairs>::kBoxA : Shape<kSingle>::kBoxA) ||
       !encode(&m.b0, a->w2, mx, a->hidden, a->dim, a->experts, hrow, 128) ||
       (pair2 && mx && (!encode_scales(&m.scales.a, p.h_scale, q.row_tiles * htiles) ||
                        !encode_scales(&m.scales.b0, a->w2_scale, weight_tiles)))))
    e = cudaErrorInvalidValue;
  if (e == cudaSuccess) {
    m.b1 = m.b0;  // (not used; the scales' map serves both tiles of a pair's 256 columns)
    m.scales.b1 = m.scales.b0;
    const int per = pair2 ? 256 : 128;
    p.scale_b[0] = a->w2_scale;
    p.a_scale = p.h_scale;
    p.k_elems = a->hidden;
    p.n_elems = a->dim;
    p.n_tiles = (a->dim + per - 1) / per;
    p.k_stages = (a->hidden + stage - 1) / stage;
    p.splits = q.splits;
    p.split_stages = q.split_stages;
    e = mx ? launch_phase<true, 2>(p, q.variant2, q.tiles2, m, s)
           : launch_phase<false, 2>(p, q.variant2, q.tiles2, m, s);
  }
  if (e == cudaSuccess && !p.direct && q.variant2 != kFew) {
    const Launch l(dim3(p.tokens, (p.dim / 4 + 127) / 128), 128, 0, s);
    e = cudaLaunchKernelEx(&l.cfg, combine, p);
  }
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "experts launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
