// dard_experts.cu - dard_experts: the products of a mixture of experts, grouped over the
// (token, slot) pairs that dard_route sorted by expert.
//
//   product<.., 1>   h = silu(w1 x) * (w3 x) of every pair, rounded (MXFP8 or bf16)
//   product<.., 2>   o = w2 h of every pair
//   combine          y_t = sum over the slots of token t of weight * o
//
// Both products are one persistent tcgen05 kernel. An output tile is 128 pairs of one expert
// (the rows of A, M = 128) by kN weight rows (B, N = kN); what a CTA computes follows from
// `offsets` alone, so no size of an expert ever travels to the host. In phase 1 the weight
// rows of a tile are kN / 2 of w1 and the same kN / 2 of w3, so that the gate and the value it
// scales meet in one thread's registers: a thread of the epilogue holds one pair (TMEM lane)
// and 32 consecutive hidden elements, which is one MX block: its scale needs no exchange.
//
// Per CTA (one per SM):
//   warps 0-7   epilogue: TMEM -> registers, then the accumulator is free for the next tile
//               while SwiGLU, the rounding and the stores run from registers;
//   warp 8      TMA producer: A rows (phase 1: gathered by token with tile::gather4, only the
//               groups of four rows that exist; phase 2: boxes of 32 consecutive rows of h),
//               B tiles, their scales (cp.async.bulk);
//   warp 9      TMEM allocation; one lane issues the scale copies (tcgen05.cp) and MMAs;
//   warp 10     phase 1, MXFP8: the scales of the gathered rows. Each lane reads 16 scale
//               bytes (four stages) of its four rows at once and writes one stage's 4 x 4
//               bytes into the tile layout.
//   Stage: 128 bytes of K of the A rows and of the B rows (128-byte swizzle), plus scales.
//   TMEM: accumulator [0, 256), scales of two stages from column 256.
//
// The work is the weights' bytes for few tokens (HBM) and the tensor pipe for many.
//
// Every wait is bounded; one that gives up sets DARD_STATUS_TIMEOUT and the CTA's abort flag,
// on which every role leaves its loop. The producer then waits (bounded) for its copies in
// flight and the issuer for its MMAs before shared memory and TMEM are released.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "dard_host.cuh"
#include "dard_internal.h"
#include "dard_mx.cuh"
#include "dard_ptx.cuh"

namespace dard {
namespace {

constexpr int kTileM = 128;            // pairs per tile
constexpr int kStageK = 128;           // bytes of K per stage
constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kProducerWarp = 8, kIssueWarp = 9, kScaleWarp = 10;
constexpr uint32_t kBytesA = kTileM * kStageK;
constexpr uint32_t kTmemAll = 512;
constexpr uint32_t kScaleCol = 256;    // first TMEM column of the scales
constexpr int kGroupM = 16;            // row tiles that share a pass over an expert's columns

struct ExpertsParams {
  const int32_t* offsets;
  const int32_t* rows;
  const int32_t* ids;
  const float* weights;
  const uint8_t* x_scale;
  const uint8_t* scale_b[2];  // phase 1: w1, w3; phase 2: w2
  uint8_t* h;                 // [row tiles * 128][hidden]
  uint8_t* h_scale;           // [row tiles][ceil(hidden / 128)][512]
  float* partial;             // [splits][pairs][dim]
  void* y;
  uint32_t* status;
  int64_t x_scale_stride, y_stride;
  long long wait_cycles;
  int32_t tokens, experts, top_k, dim, hidden, pairs;
  int32_t k_elems, n_elems;     // of this phase: reduced length, weight rows per expert
  int32_t n_tiles;              // tiles over n_elems
  int32_t k_stages;             // stages over k_elems
  int32_t splits, split_stages; // phase 2: the reduction in `splits` runs of split_stages
  int32_t max_row_tiles;        // rows of the workspace / 128
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
// Four rows r0 .. r3 (any order) from column c, one under the other in shared memory.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const void* desc, uint64_t* bar, int32_t c,
                                            int32_t r0, int32_t r1, int32_t r2, int32_t r3) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(desc)), "r"(smem_u32(bar)), "r"(c), "r"(r0), "r"(r1), "r"(r2),
      "r"(r3)
      : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}
// One 512-byte tile of scales (32 rows of 16 bytes) into four TMEM columns of every lane quarter.
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
               : "memory");
}
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::
          "r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
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

// ---------------------------------------------------------------- shapes of the two variants
// Wide: 256 weight rows per tile (one N = 256 MMA), 4 stages. Narrow: 128 weight rows, 6
// stages, twice as many tiles: for calls whose wide tiles would not fill the SMs.
template <bool kWide>
struct Shape {
  static constexpr int kN = kWide ? 256 : 128;
  static constexpr int kStages = kWide ? 4 : 6;
  static constexpr uint32_t kBytesB = kN * kStageK;
  static constexpr uint32_t kScaleA = kMxTileBytes;      // bytes of a stage's A scales
  static constexpr uint32_t kScaleB = 2 * kMxTileBytes;  // two tiles of weight scales
  static constexpr uint32_t kStage = kBytesA + kBytesB;
};

template <int kStages>
struct __align__(16) Ctl {
  uint64_t full[kStages], empty[kStages];
  uint64_t acc_full, acc_free;
  uint64_t drained;  // every MMA the issuer launched has completed
  uint32_t tmem_base;
  int32_t abort;
  int32_t first_row[DARD_MAX_EXPERTS + 1];   // offsets, clamped to [0, pairs]
  int32_t first_tile[DARD_MAX_EXPERTS + 1];  // row tiles of the experts before
};

template <bool kWide>
constexpr size_t smem_bytes() {
  using S = Shape<kWide>;
  return 1024 + static_cast<size_t>(S::kStages) * (S::kStage + S::kScaleA + S::kScaleB) +
         sizeof(Ctl<S::kStages>);
}

// One tile: pairs [row, row + count) of expert e, weight columns from n0, reduction split.
struct Tile {
  int e, row, count, row_tile, n, split;
};

// Tile `w` of the call. Within an expert, kGroupM row tiles take each column tile in turn, so
// that CTAs that run together share weights and rows in L2. `e` walks forward.
template <class C>
__device__ __forceinline__ bool get_tile(const ExpertsParams& p, const C& c, int64_t w, int& e,
                                         Tile& t) {
  const int per_row = p.n_tiles * p.splits;
  if (w >= static_cast<int64_t>(c.first_tile[p.experts]) * per_row) return false;
  while (w >= static_cast<int64_t>(c.first_tile[e + 1]) * per_row) ++e;
  const int row_tiles = c.first_tile[e + 1] - c.first_tile[e];
  const int local = static_cast<int>(w - static_cast<int64_t>(c.first_tile[e]) * per_row);
  const int group = local / (kGroupM * per_row);
  const int in_group = min(kGroupM, row_tiles - group * kGroupM);
  const int rest = local - group * kGroupM * per_row;
  const int m = group * kGroupM + rest % in_group;
  const int col = rest / in_group;
  t.e = e;
  t.n = col % p.n_tiles;
  t.split = col / p.n_tiles;
  t.row = c.first_row[e] + m * kTileM;
  t.count = min(kTileM, c.first_row[e + 1] - t.row);
  t.row_tile = c.first_tile[e] + m;
  return true;
}

__device__ __forceinline__ float silu(float g) { return __fdividef(g, 1.f + __expf(-g)); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool kMx, bool kWide, int kPhase>
__global__ void __launch_bounds__(kThreads, 1)
    product(const __grid_constant__ ExpertsParams p, const __grid_constant__ CUtensorMap map_a,
            const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_b1) {
  using S = Shape<kWide>;
  constexpr int kStages = S::kStages, kN = S::kN;
  constexpr int kElems = kMx ? 128 : 64;    // elements of K per stage
  constexpr int kStepElems = kMx ? 32 : 16; // per MMA (32 bytes)
  // weight rows of a tile from one matrix: phase 1 takes half of them from w1, half from w3
  constexpr int kCols = kPhase == 1 ? kN / 2 : kN;
  constexpr int kBoxRows = kCols < 128 ? kCols : 128;
  constexpr int kBoxes = kN / kBoxRows;     // B copies per stage
  grid_dep_launch();
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* s_scale = base + kStages * S::kStage;  // per stage: A scales, then B scales
  Ctl<kStages>& ctl = *reinterpret_cast<Ctl<kStages>*>(
      s_scale + kStages * (S::kScaleA + S::kScaleB));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long limit = p.wait_cycles > 0 ? p.wait_cycles : kWaitCycles;

  if (warp == kIssueWarp) {
    tmem_alloc<kTmemAll>(&ctl.tmem_base);
    tmem_relinquish();
  }
  if (warp == kProducerWarp && lane == 0) {
    for (int b = 0; b < kStages; ++b) {
      mbar_init(&ctl.full[b], kMx && kPhase == 1 ? 2 : 1);  // the producer (and the scale warp)
      mbar_init(&ctl.empty[b], 1);
    }
    mbar_init(&ctl.acc_full, 1);
    mbar_init(&ctl.acc_free, kEpilogueWarps);
    mbar_init(&ctl.drained, 1);
    ctl.abort = 0;
    fence_barrier_init();
    tma_prefetch_desc(&map_a);
    tma_prefetch_desc(&map_b0);
    if (kPhase == 1) tma_prefetch_desc(&map_b1);
  }
  // (offsets were complete before this call's first kernel began)
  for (int i = threadIdx.x; i <= p.experts; i += kThreads)
    ctl.first_row[i] = min(max(p.offsets[i], 0), p.pairs);
  __syncthreads();
  if (warp == 0) {  // row tiles before each expert
    int carry = 0;
    for (int b = 0; b < p.experts; b += 32) {
      const int i = b + lane;
      const int n = i < p.experts ? max(ctl.first_row[i + 1] - ctl.first_row[i], 0) : 0;
      int s = (n + kTileM - 1) / kTileM;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
      }
      // a plan that is none (offsets that fall) never reaches past the workspace
      if (i < p.experts) ctl.first_tile[i + 1] = min(carry + s, p.max_row_tiles);
      carry = min(carry + __shfl_sync(0xffffffffu, s, 31), p.max_row_tiles);
    }
    if (lane == 0) ctl.first_tile[0] = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem_base;
  volatile int32_t* abort_flag = &ctl.abort;
  const auto give_up = [&]() {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, DARD_STATUS_TIMEOUT);
  };
  const int split_stages = kPhase == 2 ? p.split_stages : p.k_stages;

  if (warp == kProducerWarp) {
    // -------------------------------------------------------------- TMA producer
    int e = 0, use = 0;
    bool ok = true;
    Tile t;
    if (kPhase == 2) grid_dep_wait();  // h is complete
    for (int64_t w = blockIdx.x; ok && get_tile(p, ctl, w, e, t); w += gridDim.x) {
      int r[4];  // phase 1: tokens of this lane's four rows (a row index past the end reads 0)
      uint32_t bytes_a;
      if (kPhase == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = 4 * lane + i;
          const int pair = at < t.count ? __ldg(p.rows + t.row + at) : -1;
          r[i] = pair >= 0 && pair < p.pairs ? pair / p.top_k : p.tokens;
        }
        bytes_a = (t.count + 3) / 4 * 4 * kStageK;
      } else {
        bytes_a = (t.count + 31) / 32 * 32 * kStageK;
      }
      const int k0 = t.split * split_stages, k1 = min(p.k_stages, k0 + split_stages);
      const int n0 = t.n * kCols;
      uint32_t scale_bytes = 0;
      if (kMx) {
        // phase 2: a second tile of weight scales where the tile has more than 128 rows
        scale_bytes = kPhase == 1 ? 2 * kMxTileBytes
                                  : kMxTileBytes * (kN > 128 && n0 + 128 < p.n_elems ? 3 : 2);
      }
      for (int k = k0; k < k1; ++k, ++use) {
        const int b = use % kStages;
        ok = !*abort_flag && (use < kStages ||
                              mbar_wait(&ctl.empty[b], ((use / kStages) - 1) & 1, limit));
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        uint8_t* sa = base + b * S::kStage;
        uint8_t* sb = sa + kBytesA;
        uint8_t* ss = s_scale + b * (S::kScaleA + S::kScaleB);
        if (lane == 0) mbar_arrive_expect_tx(&ctl.full[b], bytes_a + S::kBytesB + scale_bytes);
        __syncwarp();
        if (kPhase == 1) {
          if (4 * lane < t.count)
            tma_gather4(smem_u32(sa) + lane * 4 * kStageK, &map_a, &ctl.full[b], k * kElems, r[0],
                        r[1], r[2], r[3]);
        } else if (32 * lane < t.count) {
          tma_load_2d(sa + lane * 32 * kStageK, &map_a, &ctl.full[b], k * kElems,
                      t.row_tile * kTileM + 32 * lane);
        }
        if (lane < kBoxes && use != p.test_drop) {
          const int col = kPhase == 1 ? n0 : n0 + lane * kBoxRows;
          tma_load_3d(sb + lane * kBoxRows * kStageK, kPhase == 1 && lane == 1 ? &map_b1 : &map_b0,
                      &ctl.full[b], k * kElems, col, t.e);
        }
        if (kMx && lane == 0) {
          const int row_tiles = (p.n_elems + 127) / 128;
          const int64_t at = (static_cast<int64_t>(t.e) * row_tiles + n0 / 128) * p.k_stages + k;
          if (kPhase == 1) {
            bulk_load(ss + S::kScaleA, p.scale_b[0] + at * kMxTileBytes, kMxTileBytes, &ctl.full[b]);
            bulk_load(ss + S::kScaleA + kMxTileBytes, p.scale_b[1] + at * kMxTileBytes, kMxTileBytes,
                      &ctl.full[b]);
          } else {
            bulk_load(ss, p.h_scale + (static_cast<int64_t>(t.row_tile) * p.k_stages + k) * kMxTileBytes,
                      kMxTileBytes, &ctl.full[b]);
            bulk_load(ss + S::kScaleA, p.scale_b[0] + at * kMxTileBytes, kMxTileBytes, &ctl.full[b]);
            if (kN > 128 && n0 + 128 < p.n_elems)
              bulk_load(ss + S::kScaleA + kMxTileBytes,
                        p.scale_b[0] + (at + p.k_stages) * kMxTileBytes, kMxTileBytes, &ctl.full[b]);
          }
        }
      }
    }
    if (!ok) {
      if (lane == 0) give_up();
      // copies in flight land before shared memory is released: the last use of each stage
      for (int u = max(0, use - kStages); u < use; ++u)
        mbar_wait(&ctl.full[u % kStages], (u / kStages) & 1, limit);
    }
    __syncwarp();
  } else if (warp == kIssueWarp) {
    // -------------------------------------------------------------- MMA issuer
    if (lane == 0) {
      int e = 0, use = 0, tiles = 0;
      bool ok = true;
      Tile t;
      for (int64_t w = blockIdx.x; ok && get_tile(p, ctl, w, e, t); w += gridDim.x, ++tiles) {
        ok = tiles == 0 || mbar_wait(&ctl.acc_free, (tiles - 1) & 1, limit);
        if (!ok) break;
        tc_fence_after();
        const int k0 = t.split * split_stages, k1 = min(p.k_stages, k0 + split_stages);
        // narrow phase 1: a tile's 64 weight rows are half of a tile of 128 scales
        const uint32_t half = kPhase == 1 && kCols == 64 ? (t.n & 1) * 2 : 0;
        for (int k = k0; k < k1; ++k, ++use) {
          const int b = use % kStages;
          ok = !*abort_flag && mbar_wait(&ctl.full[b], (use / kStages) & 1, limit);
          if (!ok) break;
          tc_fence_after();
          const uint32_t sa = smem_u32(base + b * S::kStage), sb = sa + kBytesA;
          const uint32_t sfa = tmem + kScaleCol + (use & 1) * 16, sfb = sfa + 8;
          if (kMx) {
            const uint32_t ss = smem_u32(s_scale + b * (S::kScaleA + S::kScaleB));
            copy_scales(sfa, scale_desc(ss));
            copy_scales(sfb, scale_desc(ss + S::kScaleA));
            if (kPhase == 1 || kN > 128) copy_scales(sfb + 4, scale_desc(ss + S::kScaleA + kMxTileBytes));
          }
          const int steps = min(4, (p.k_elems - k * kElems + kStepElems - 1) / kStepElems);
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            if (ks >= steps) break;
            const uint32_t acc = (k > k0 || ks > 0) ? 1u : 0u;
            const uint64_t da = smem_desc_sw128(sa + ks * 32, 16, 1024);
            const uint64_t db = smem_desc_sw128(sb + ks * 32, 16, 1024);
            if constexpr (!kMx) {
              mma_ss(tmem, da, db, idesc_bf16_f32(kTileM, kN, 0, 0), acc);
            } else if constexpr (kPhase == 1 && kCols == 64) {
              // w1's and w3's scales lie in different tiles: one MMA for each
              mma_mx(tmem, da, db, idesc_mx(kTileM, 64, ks), sfa, sfb + half, acc);
              mma_mx(tmem + 64, da, smem_desc_sw128(sb + 64 * kStageK + ks * 32, 16, 1024),
                     idesc_mx(kTileM, 64, ks), sfa, sfb + 4 + half, acc);
            } else {
              mma_mx(tmem, da, db, idesc_mx(kTileM, kN, ks), sfa, sfb, acc);
            }
          }
          mma_commit(&ctl.empty[b]);
        }
        if (ok) mma_commit(&ctl.acc_full);
      }
      if (!ok) give_up();
      mma_commit(&ctl.drained);
    }
    __syncwarp();
  } else if (warp == kScaleWarp) {
    // -------------------------------------------------------------- scales of gathered rows
    if (kMx && kPhase == 1) {
      int e = 0, use = 0;
      bool ok = true;
      Tile t;
      for (int64_t w = blockIdx.x; ok && get_tile(p, ctl, w, e, t); w += gridDim.x) {
        // lane l: rows l, 32 + l, 64 + l, 96 + l, whose words lie side by side in the tile
        const uint4* src[4];
        uint32_t now[4][4], ahead[4][4];  // [row][stage within a group of four]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = 32 * i + lane;
          const int pair = at < t.count ? __ldg(p.rows + t.row + at) : -1;
          src[i] = pair >= 0 && pair < p.pairs
                       ? reinterpret_cast<const uint4*>(
                             p.x_scale + static_cast<int64_t>(pair / p.top_k) * p.x_scale_stride)
                       : nullptr;
        }
        const auto fetch = [&](int group, uint32_t (&d)[4][4]) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (src[i] != nullptr && 4 * group < p.k_stages) v = __ldg(src[i] + group);
            d[i][0] = v.x;
            d[i][1] = v.y;
            d[i][2] = v.z;
            d[i][3] = v.w;
          }
        };
        fetch(0, ahead);
        for (int k = 0; ok && k < p.k_stages; k += 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) now[i][j] = ahead[i][j];
          }
          fetch(k / 4 + 1, ahead);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (k + j >= p.k_stages) break;
            const int b = use % kStages;
            ok = !*abort_flag && (use < kStages ||
                                  mbar_wait(&ctl.empty[b], ((use / kStages) - 1) & 1, limit));
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            uint8_t* ss = s_scale + b * (S::kScaleA + S::kScaleB);
            reinterpret_cast<uint4*>(ss)[lane] = make_uint4(now[0][j], now[1][j], now[2][j], now[3][j]);
            fence_proxy_async_smem();  // before the tensor core's copy reads them
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.full[b]);
            ++use;
          }
        }
      }
      if (!ok && lane == 0) give_up();
      __syncwarp();
    }
  } else if (warp < kEpilogueWarps) {
    // -------------------------------------------------------------- epilogue
    const int quarter = warp & 3, half = warp >> 2;
    const int r = quarter * 32 + lane;  // TMEM lane = row of the tile
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    constexpr int kChunks = kN / 2 / 32;  // 32-column loads of a warp: half of the tile
    int e = 0, tiles = 0;
    bool ok = true;
    Tile t;
    if (kPhase == 2) {
      grid_dep_wait();
      if (p.direct) {
        // tokens without an expert: no pair of theirs reaches any tile
        constexpr int kRun = 32 * kEpilogueWarps;
        for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRun + warp * 32; t0 < p.tokens;
             t0 += static_cast<int64_t>(gridDim.x) * kRun) {
          uint32_t missing = __ballot_sync(
              0xffffffffu, t0 + lane < p.tokens && p.ids[t0 + lane] < 0);
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
    for (int64_t w = blockIdx.x; ok && get_tile(p, ctl, w, e, t); w += gridDim.x, ++tiles) {
      const bool in = r < t.count;
      int pair = 0;
      if (kPhase == 2) pair = in ? __ldg(p.rows + t.row + r) : -1;
      ok = !*abort_flag && mbar_wait(&ctl.acc_full, tiles & 1, limit);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
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
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.acc_free);
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
              uint4* dst = reinterpret_cast<uint4*>(p.h + row * p.hidden + col);
              dst[0] = make_uint4(q[0], q[1], q[2], q[3]);
              dst[1] = make_uint4(q[4], q[5], q[6], q[7]);
              const int tiles_h = (p.hidden + 127) / 128;
              p.h_scale[(static_cast<int64_t>(t.row_tile) * tiles_h + col / 128) * kMxTileBytes +
                        mx_tile_byte(r, col / 32)] = static_cast<uint8_t>(b);
            }
          } else if (in && col < p.hidden) {
            uint4* dst = reinterpret_cast<uint4*>(p.h + (row * p.hidden + col) * 2);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dst[i] = make_uint4(pack2(v[8 * i], v[8 * i + 1]), pack2(v[8 * i + 2], v[8 * i + 3]),
                                  pack2(v[8 * i + 4], v[8 * i + 5]), pack2(v[8 * i + 6], v[8 * i + 7]));
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
          if (p.direct && !p.y_f32) {
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
            float* to = p.direct ? static_cast<float*>(p.y) + pair * p.y_stride + col
                                 : p.partial + (static_cast<int64_t>(t.split) * p.pairs + pair) * p.dim + col;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              reinterpret_cast<float4*>(to)[i] =
                  make_float4(__uint_as_float(a[4 * i]) * weight, __uint_as_float(a[4 * i + 1]) * weight,
                              __uint_as_float(a[4 * i + 2]) * weight,
                              __uint_as_float(a[4 * i + 3]) * weight);
          }
        }
      }
    }
    if (!ok && lane == 0) give_up();
    __syncwarp();
  }
  // ---------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    if (!mbar_wait(&ctl.drained, 0, limit) && lane == 0) give_up();
    __syncwarp();
    tc_fence_after();
    tmem_dealloc<kTmemAll>(tmem);
  }
}

// y_t = sum over slots (in order) of weight * (sum over splits of partial). Eight columns per
// thread.
template <typename Y>
__global__ void __launch_bounds__(128) combine(const __grid_constant__ ExpertsParams p) {
  grid_dep_wait();
  const int64_t t = blockIdx.x;
  for (int col = 8 * (blockIdx.y * 128 + threadIdx.x); col < p.dim; col += 8 * 128 * gridDim.y) {
    float sum[8] = {};
    for (int s = 0; s < p.top_k; ++s) {
      const int64_t pair = t * p.top_k + s;
      if (p.ids[pair] < 0) continue;
      const float w = p.weights[pair];
      float o[8] = {};
      for (int i = 0; i < p.splits; ++i) {
        const float4* src = reinterpret_cast<const float4*>(
            p.partial + (static_cast<int64_t>(i) * p.pairs + pair) * p.dim + col);
        const float4 a = src[0], b = src[1];
        o[0] += a.x; o[1] += a.y; o[2] += a.z; o[3] += a.w;
        o[4] += b.x; o[5] += b.y; o[6] += b.z; o[7] += b.w;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, o[i], sum[i]);
    }
    Y* y = static_cast<Y*>(p.y) + t * p.y_stride + col;
    if constexpr (sizeof(Y) == 2) {
      *reinterpret_cast<uint4*>(y) = make_uint4(pack2(sum[0], sum[1]), pack2(sum[2], sum[3]),
                                                pack2(sum[4], sum[5]), pack2(sum[6], sum[7]));
    } else {
      reinterpret_cast<float4*>(y)[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
      reinterpret_cast<float4*>(y)[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
    }
  }
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

template <bool kMx, bool kWide, int kPhase>
cudaError_t launch_product(const ExpertsParams& p, int64_t tiles, const CUtensorMap& a,
                           const CUtensorMap& b0, const CUtensorMap& b1, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const size_t smem = smem_bytes<kWide>();
  const cudaError_t e = ensure_smem_attr(product<kMx, kWide, kPhase>, smem, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(std::min<int64_t>(tiles, sm_count())));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kPhase == 2 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, product<kMx, kWide, kPhase>, p, a, b0, b1);
}

template <bool kMx, int kPhase>
cudaError_t launch_phase(const ExpertsParams& p, bool wide, int64_t tiles, const CUtensorMap& a,
                         const CUtensorMap& b0, const CUtensorMap& b1, cudaStream_t s) {
  return wide ? launch_product<kMx, true, kPhase>(p, tiles, a, b0, b1, s)
              : launch_product<kMx, false, kPhase>(p, tiles, a, b0, b1, s);
}

template <typename Y>
cudaError_t launch_combine(const ExpertsParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.tokens, (p.dim / 8 + 127) / 128);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, combine<Y>, p);
}

constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Sizes that follow from a call's sizes alone.
struct Plan {
  int64_t pairs, row_tiles;  // at most so many row tiles of 128 pairs
  bool wide1, wide2;
  int64_t tiles1, tiles2;    // at most so many tiles of each phase
  int splits, split_stages;
  size_t h_bytes, h_scale_bytes, partial_bytes;
};

// Wide tiles unless they would leave SMs idle (their count, over the row tiles that the call
// can have, is below the SM count): a narrow tile reads its rows for half as many weight
// rows. Where even narrow tiles of phase 2 leave SMs idle (few pairs, a long reduction), the
// reduction is split, into runs of at least four stages.
Plan make_plan(int64_t tokens, int experts, int top_k, int dim, int hidden, bool mx) {
  Plan q = {};
  q.pairs = tokens * top_k;
  q.row_tiles = q.pairs / kTileM + std::min<int64_t>(experts, q.pairs);
  const int64_t sms = sm_count();
  const auto tiles = [&](int n, int per) { return q.row_tiles * ((n + per - 1) / per); };
  q.wide1 = tiles(hidden, 128) >= sms;
  q.wide2 = tiles(dim, 256) >= sms;
  q.tiles1 = tiles(hidden, q.wide1 ? 128 : 64);
  q.tiles2 = tiles(dim, q.wide2 ? 256 : 128);
  const int stages = (hidden + (mx ? 127 : 63)) / (mx ? 128 : 64);
  int64_t splits = 1;
  if (q.tiles2 * 2 <= sms) splits = std::max<int64_t>(1, std::min<int64_t>(sms / q.tiles2, stages / 4));
  q.split_stages = static_cast<int>((stages + splits - 1) / splits);
  q.splits = (stages + q.split_stages - 1) / q.split_stages;
  q.tiles2 *= q.splits;
  const size_t rows = static_cast<size_t>(q.row_tiles) * kTileM;
  q.h_bytes = up256(rows * hidden * (mx ? 1 : 2));
  q.h_scale_bytes = mx ? up256(static_cast<size_t>(q.row_tiles) * ((hidden + 127) / 128) * kMxTileBytes) : 0;
  const bool direct = top_k == 1 && q.splits == 1;
  q.partial_bytes = direct ? 0 : up256(static_cast<size_t>(q.splits) * q.pairs * dim * 4);
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
  size_t most = 0;
  for (int mx = 0; mx < 2; ++mx) {
    const Plan q = make_plan(tokens, experts, top_k, dim, hidden, mx != 0);
    most = std::max(most, q.h_bytes + q.h_scale_bytes + q.partial_bytes);
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
  const size_t need = q.h_bytes + q.h_scale_bytes + q.partial_bytes;
  if (!a->workspace || a->workspace_bytes < need)
    return report(DARD_ERR_WORKSPACE, "workspace of %zu bytes needed", need);
  if (!aligned(a->workspace, 256)) return report(DARD_ERR_ALIGN, "workspace must be 256-byte aligned");

  ExpertsParams p = {};
  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  p.offsets = a->offsets;
  p.rows = a->rows;
  p.ids = a->ids;
  p.weights = a->weights;
  p.x_scale = a->x_scale;
  p.scale_b[0] = a->w1_scale;
  p.scale_b[1] = a->w3_scale;
  p.h = ws;
  p.h_scale = ws + q.h_bytes;
  p.partial = reinterpret_cast<float*>(ws + q.h_bytes + q.h_scale_bytes);
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
  p.direct = q.partial_bytes == 0;
  p.test_drop = -1;
  // Test hooks (failure-path tests; unset in normal operation): a wait bound, and a stage whose
  // weights never arrive.
  if (const char* w = std::getenv("DARD_TEST_WAIT_CYCLES")) p.wait_cycles = std::atoll(w);
  if (const char* d = std::getenv("DARD_TEST_DROP_KV")) p.test_drop = std::atoi(d);

  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int stage = mx ? 128 : 64;
  cudaError_t e = std::getenv("DARD_TEST_FAIL_LAUNCH") ? cudaErrorLaunchFailure : cudaSuccess;
  CUtensorMap ma, mb0, mb1;
  // phase 1: rows of x by token, rows of w1 and w3
  const uint64_t drow = static_cast<uint64_t>(a->dim) * esz, hrow = static_cast<uint64_t>(a->hidden) * esz;
  const uint32_t box1 = q.wide1 ? 128 : 64;
  if (e == cudaSuccess &&
      (!encode(&ma, a->x, mx, a->dim, a->tokens, 0, a->x_stride * esz, 1) ||
       !encode(&mb0, a->w1, mx, a->dim, a->hidden, a->experts, drow, box1) ||
       !encode(&mb1, a->w3, mx, a->dim, a->hidden, a->experts, drow, box1)))
    e = cudaErrorInvalidValue;
  if (e == cudaSuccess) {
    p.k_elems = a->dim;
    p.n_elems = a->hidden;
    p.n_tiles = (a->hidden + box1 - 1) / box1;
    p.k_stages = (a->dim + stage - 1) / stage;
    p.splits = 1;
    p.split_stages = p.k_stages;
    e = mx ? launch_phase<true, 1>(p, q.wide1, q.tiles1, ma, mb0, mb1, s)
           : launch_phase<false, 1>(p, q.wide1, q.tiles1, ma, mb0, mb1, s);
  }
  // phase 2: rows of h, rows of w2
  if (e == cudaSuccess &&
      (!encode(&ma, p.h, mx, a->hidden, static_cast<uint64_t>(q.row_tiles) * kTileM, 0, hrow, 32) ||
       !encode(&mb0, a->w2, mx, a->hidden, a->dim, a->experts, hrow, 128)))
    e = cudaErrorInvalidValue;
  if (e == cudaSuccess) {
    const int per = q.wide2 ? 256 : 128;
    p.scale_b[0] = a->w2_scale;
    p.k_elems = a->hidden;
    p.n_elems = a->dim;
    p.n_tiles = (a->dim + per - 1) / per;
    p.k_stages = (a->hidden + stage - 1) / stage;
    p.splits = q.splits;
    p.split_stages = q.split_stages;
    e = mx ? launch_phase<true, 2>(p, q.wide2, q.tiles2, ma, mb0, mb0, s)
           : launch_phase<false, 2>(p, q.wide2, q.tiles2, ma, mb0, mb0, s);
  }
  if (e == cudaSuccess && !p.direct)
    e = p.y_f32 ? launch_combine<float>(p, s) : launch_combine<__nv_bfloat16>(p, s);
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "experts launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
