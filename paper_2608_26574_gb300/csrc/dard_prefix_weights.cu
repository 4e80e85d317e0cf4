// dard_prefix_weights.cu - the attention weight that each key of a shared prefix has received
// (dard_prefix_weights): per key/value head g and key j the sum over the query rows and the heads
// of the group of exp(c <q, k_j> - lse). Validation, the bf16 kernel on the tensor cores, the fp32
// kernel on CUDA cores, and the kernel that adds up the parts of a split.
//
// weights_tc: 128 keys of one key/value head stay in TMEM as the A operand (their rows read straight
// from global memory); tiles of up to 128 (row, head) queries pass by as B, so that an accumulator row
// is a key and a thread adds up its key's exponentials along the row: no reduction across threads
// until the end, no atomics, one order of addition. 28 warps:
//   warps 0-23 exponentials and sums: groups of eight warps take every third tile; of a group, warps q
//              and q + 4 share TMEM lane quarter q (keys 32q .. 32q + 31), each taking 64 of the 128
//              queries;
//   warp 24    TMA producer: Q through 6 stages (128-element heads: 192 KB);
//   warp 25    TMEM allocator and issuer: S_j = K Q_j^T into a buffer of 128 columns for each group;
//   warps 26, 27 the queries' normalisers through 6 stages, every other tile each (one warp took 800
//              cycles a tile, more than the products do).
// TMEM: S ring [0, 384), K [448, 448 + D/2). Bound by the issue slots of the exponentials and by TMEM,
// which the products' A operand and the workers' reads share: about 915 cycles per 128 x 128 scores, of
// which the tensor cores work 512. Measured: 4608 rows of 28 heads on 4 of 128 over 32768 keys 850-990 us
// (1090-1270 TFLOP/s; the more, the more sums exact_sum32 forms again; 688 without the exponentials); with K
// in shared memory 960 instead of 870.
// Each tile's sum is formed on its own and then added to the key's total (two levels: the
// rounding of a long sum grows with the number of tiles, not of queries).
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "dard_prefix.cuh"

namespace dard {
namespace {

struct WeightsParams {
  const void* q;
  const float* lse;
  const void* pk;
  const float* w_in;
  float* w;
  float* part;               // [nsplit][hkv][prefix_len], nsplit > 1
  uint32_t* status;
  int64_t row_stride, head_stride, w_in_stride, w_stride;
  int32_t rows, hq, hkv, prefix_len, group;
  int32_t box_heads, box_rows, head_blocks;  // a query tile: box_rows rows x box_heads heads
  int32_t q_tiles, key_tiles, nsplit;
  float scale_log2, decay;
  float large;               // bf16: sums of 32 columns above it are formed again (exact_sum32)
  float lse_hi, lse_lo;      // what lse is multiplied with, in two parts
  double scale;              // of the scores, times log2 e: scale_log2 before its rounding
  long long wait_cycles;
  int32_t test_drop_kv;
};

constexpr float kLog2e = 1.4426950408889634f;

// -lse in the unit in which scale_log2 takes the scores.
__device__ __forceinline__ float lse_unit(const WeightsParams& p, float lse) {
  return fabsf(lse) == INFINITY ? -lse : fmaf(lse, p.lse_hi, lse * p.lse_lo);
}

// Adds what the earlier sum contributes.
__device__ __forceinline__ float with_earlier(const WeightsParams& p, int g, int key, float sum) {
  return p.w_in ? fmaf(p.decay, p.w_in[g * p.w_in_stride + key], sum) : sum;
}

// ---------------------------------------------------------------- bf16, tensor cores
constexpr int kThreads = 896;
constexpr int kGroups = 3;
constexpr int kQStages = 6, kSBufs = kGroups;
static_assert(kQStages % kGroups == 0, "a group's tiles come back to the stages that it used");
constexpr int kWorkers = 8;  // warps of a tile
constexpr int kWProd = 24, kWMma = 25, kWLse = 26;
constexpr uint32_t kKCol = 448;  // TMEM columns of K

struct __align__(16) Ctl {
  uint64_t k_full;  // K is in TMEM
  uint64_t q_full[kQStages], q_empty[kQStages];
  uint64_t l_full[kQStages], l_empty[kQStages];
  uint64_t s_full[kSBufs], s_free[kSBufs];
  uint64_t drained;
  uint32_t tmem_base;
  int32_t abort;
  int32_t odd_keys;               // an element of K is not finite (before k_full)
  __align__(16) float lse[kQStages][kBM];  // times -log2 e (read four at a time)
  uint32_t off[kQStages][4];      // queries that add nothing (bit per column)
  float red[2 * kGroups][kBM];
};

template <int D>
constexpr size_t smem_bytes() {
  return 1024 + kQStages * static_cast<size_t>(kTN) * D * 2 + sizeof(Ctl);
}

__device__ __forceinline__ void flag_timeout(const WeightsParams& p, Ctl& ctl) {
  ctl.abort = 1;
  if (p.status) atomicOr(p.status, DARD_STATUS_TIMEOUT);
}

// Sum over 32 columns of 2^(s sl - lse) for one key. kOff: columns with a bit of `off` count for
// nothing, whatever their scores are.
template <bool kOff>
__device__ __forceinline__ float sum32(const uint32_t (&s)[32], const float* lse, uint32_t off,
                                       uint64_t sl2) {
  uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const ulonglong2 n = *reinterpret_cast<const ulonglong2*>(lse + 4 * e);
    float x[4];
    f2_unpack(f2_fma(f2_pack(__uint_as_float(s[4 * e]), __uint_as_float(s[4 * e + 1])), sl2, n.x), x[0], x[1]);
    f2_unpack(f2_fma(f2_pack(__uint_as_float(s[4 * e + 2]), __uint_as_float(s[4 * e + 3])), sl2, n.y), x[2], x[3]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = ex2_approx(x[k]);
      if (kOff && (off >> (4 * e + k) & 1u)) x[k] = 0.f;
    }
    acc[(2 * e) & 3] = f2_add(acc[(2 * e) & 3], f2_pack(x[0], x[1]));
    acc[(2 * e + 1) & 3] = f2_add(acc[(2 * e + 1) & 3], f2_pack(x[2], x[3]));
  }
  float a, b;
  f2_unpack(f2_add(f2_add(acc[0], acc[1]), f2_add(acc[2], acc[3])), a, b);
  return a + b;
}

// Sums above p.large (some lane's of the warp) once more, with exact scores: the tensor cores cut the bits that
// a running sum has no room for, which takes up to two units in the last place off a large score, 3.4e-6 of
// its exponential at a score of 35 and more where small products follow large ones. p.large is a quarter of
// the columns, whatever the prefix: keys that draw that much of their queries' weight reach it, and where lse is
// over other keys (a part of them, a cache that has changed since) single terms may be as large as they like, and
// are a key's whole sum. Such a key costs one of its CTA's warps 2 to 3 us for every 32 queries. Key by key for
// those that need it, a lane for each of the 32 columns from `first` on; eight products at a time, their sums added up
// with what the roundings cut off. 4608 rows of 28 heads over 32768 keys: 842 us without it, 845-850 while no
// sum is that large, 887-983 with lse over 256 of the keys, where the largest error against 64 bits goes from
// 3.8e-6 to 0.6e-6 (above all of the columns 868-931, an eighth 901-1018); one row over 4096 keys 8 instead
// of 6 us. A key that takes half of every query's weight makes its CTA form nearly every sum again: 4608 rows over
// 4096 keys 123 -> 690 us, over 32768 keys 851 -> 1283, 64 rows over 4096 8 -> 19. Not inlined: the loop that calls it has no
// register to spare (inlined 1630 us).
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {  // bf16 pairs
  c = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), c);
  return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), c);
}
template <int D>
__device__ __noinline__ float exact_sum32(const WeightsParams& p, float sum, int g, int key, int tile, int first) {
  const int lane = threadIdx.x & 31, c = first + lane;
  const int row = tile / p.head_blocks * p.box_rows + c / p.box_heads;
  const int head = tile % p.head_blocks * p.box_heads + c % p.box_heads;  // of the group
  const bool in = c < p.box_rows * p.box_heads && row < p.rows && head < p.group;
  const int64_t query = static_cast<int64_t>(row) * p.hq + g * p.group + head;  // this lane's, if it is one
  const float lse = in ? __ldg(p.lse + query) : INFINITY;
  for (uint32_t lanes = __ballot_sync(0xffffffffu, sum > p.large && key < p.prefix_len); lanes; lanes &= lanes - 1) {
    const int of = __ffs(lanes) - 1;
    const int at = __shfl_sync(0xffffffffu, key, of);
    float x = 0.f;
    if (in) {
      const uint4* k = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.pk) + at * p.row_stride +
                                                      g * p.head_stride);
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + query * D);
      float z = 0.f, left = 0.f;  // the sum, and what its roundings have left out
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        const uint4 u = __ldg(k + i), v = __ldg(q + i);
        const float dot = dot2(u.x, v.x, dot2(u.y, v.y, dot2(u.z, v.z, dot2(u.w, v.w, 0.f))));
        const float to = z + dot, added = to - z;
        left += (z - (to - added)) + (dot - added);
        z = to;
      }
      if (left != left) left = 0.f;  // (z is infinite)
      // (with lse = +inf q may hold anything)
      if (lse != INFINITY)
        x = ex2_approx(static_cast<float>((static_cast<double>(z) + left) * p.scale - lse * 1.4426950408889634));
    }
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) x += __shfl_xor_sync(0xffffffffu, x, i);
    if (lane == of) sum = x;
  }
  return sum;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    weights_tc(const __grid_constant__ WeightsParams p, const __grid_constant__ CUtensorMap tq) {
  constexpr int kSub = D / 64;
  constexpr uint32_t kKSub = kTN * 128;
  constexpr uint32_t kTile = kSub * kKSub;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* sQ = base;
  Ctl& ctl = *reinterpret_cast<Ctl*>(sQ + kQStages * kTile);
  grid_dep_launch();
  const int item = blockIdx.x / p.nsplit, part = blockIdx.x % p.nsplit;
  const int g = item / p.key_tiles, key0 = item % p.key_tiles * kTN;
  const int j0 = static_cast<int>(static_cast<long long>(p.q_tiles) * part / p.nsplit);
  const int n = static_cast<int>(static_cast<long long>(p.q_tiles) * (part + 1) / p.nsplit) - j0;
  // (a shuffle's result is the warp's, as the compiler knows, and so are the branches on it: 866 -> 842 us)
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const long long wlim = p.wait_cycles > 0 ? p.wait_cycles : kWaitCycles;
  const int columns = p.box_heads * p.box_rows;  // queries of a tile, at most 128

  if (warp == kWProd && lane == 0) {
    mbar_init(&ctl.k_full, 16);
    mbar_init(&ctl.drained, 1);
    for (int b = 0; b < kQStages; ++b) {
      mbar_init(&ctl.q_full[b], 1);
      mbar_init(&ctl.q_empty[b], 1);
      mbar_init(&ctl.l_full[b], 1);
      mbar_init(&ctl.l_empty[b], kWorkers);
    }
    for (int b = 0; b < kSBufs; ++b) {
      mbar_init(&ctl.s_full[b], 1);
      mbar_init(&ctl.s_free[b], kWorkers);
    }
    ctl.abort = 0;
    ctl.odd_keys = 0;
    fence_barrier_init();
  }
  if (warp == kWMma) {
    tmem_alloc<kTmemCols>(&ctl.tmem_base);
    tmem_relinquish();
  }
  uint32_t kreg[D / 8];  // workers: a quarter of key 32 (warp % 4) + lane's row
  if (warp < 16) {
    const int key = key0 + (warp & 3) * 32 + lane;
    const uint4* src = reinterpret_cast<const uint4*>(
        static_cast<const __nv_bfloat16*>(p.pk) + (key < p.prefix_len ? key * p.row_stride + g * p.head_stride : 0) +
        (warp >> 2) * (D / 4));
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const uint4 u = key < p.prefix_len ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
      kreg[4 * c] = u.x;
      kreg[4 * c + 1] = u.y;
      kreg[4 * c + 2] = u.z;
      kreg[4 * c + 3] = u.w;
    }
  }
  // rows of the stages that no copy writes: zeros, whose scores (0; NaN with a key that is not finite) count for
  // nothing with lse = +inf
  for (int i = columns * 8 + threadIdx.x; i < kTN * 8; i += kThreads)
    for (int b = 0; b < min(n, kQStages) * kSub; ++b)
      *reinterpret_cast<uint4*>(sQ + b * kKSub + 16 * i) = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  volatile int32_t* abort_flag = &ctl.abort;

  if (warp == kWProd) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int last = -1;
      for (int j = 0; j < n && !*abort_flag; ++j) {
        const int b = j % kQStages;
        if (j >= kQStages && !mbar_wait(&ctl.q_empty[b], ((j - kQStages) / kQStages) & 1, wlim)) {
          flag_timeout(p, ctl);
          break;
        }
        const int tile = j0 + j;
        const int head = g * p.group + tile % p.head_blocks * p.box_heads;
        const int row = tile / p.head_blocks * p.box_rows;
        mbar_arrive_expect_tx(&ctl.q_full[b], kSub * columns * 128);
        if (j != p.test_drop_kv)  // (test hook: this copy is never issued)
          for (int s = 0; s < kSub; ++s)
            tma_load_3d(sQ + b * kTile + s * kKSub, &tq, &ctl.q_full[b], s * 64, head, row);
        last = j;
      }
      // every copy issued lands before shared memory is released: the latest use of each stage
      for (int b = 0; b < kQStages; ++b) {
        const int jb = last - ((last - b) % kQStages + kQStages) % kQStages;
        if (last >= 0 && jb >= 0 && jb != p.test_drop_kv)
          mbar_wait(&ctl.q_full[b], (jb / kQStages) & 1, wlim);
      }
    }
  } else if (warp == kWMma) {
    // ------------------------------------------------------------ issuer
    // (the whole warp walks the loop, so that what it computes is uniform over the warp and stays in
    // uniform registers; one elected lane issues: with one lane walking alone a tile took 1600
    // cycles, most of them the issue of its products)
    constexpr uint32_t kId = idesc_bf16_f32(kBM, kTN, 0, 0);
    const bool issue = elect_one();
    const uint64_t dq = smem_desc_sw128(smem_u32(sQ), 16, 1024);
    const uint32_t tK = ctl.tmem_base + kKCol;
    bool ok = warp_wait(&ctl.k_full, 0, wlim);
    for (int j = 0; j < n && ok; ++j) {
      const int b = j % kQStages, sb = j % kSBufs;
      if (j >= kSBufs) ok = warp_wait(&ctl.s_free[sb], ((j - kSBufs) / kSBufs) & 1, wlim);
      ok = ok && warp_wait(&ctl.q_full[b], (j / kQStages) & 1, wlim);
      if (!ok) break;
      tc_fence_after();
      if (issue) {
        const uint64_t db = dq + b * (kTile / 16);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          mma_ts(ctl.tmem_base + sb * kTN, tK + ks * 8, db + (ks >> 2) * (kKSub / 16) + (ks & 3) * 2, kId, ks > 0);
        mma_commit(&ctl.s_full[sb]);
        mma_commit(&ctl.q_empty[b]);
      }
    }
    if (!ok && lane == 0) flag_timeout(p, ctl);
    if (issue) mma_commit(&ctl.drained);
    __syncwarp();
  } else if (warp >= kWLse) {
    // ------------------------------------------------------------ normalisers
    // (two tiles' loads in flight; column 32 e + lane of a tile is row rr[e] of it, `at[e]` elements on)
    int rr[4], at[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = 32 * e + lane, h = c % p.box_heads;
      rr[e] = c < columns ? c / p.box_heads : INT_MAX;  // (no column: behind the last row)
      at[e] = c / p.box_heads * p.hq + h;
    }
    auto fetch = [&](int j, float (&v)[4]) {
      const int tile = j0 + j;
      int row0 = tile * p.box_rows, h0 = 0;
      if (p.head_blocks > 1) {
        h0 = tile % p.head_blocks * p.box_heads;
        row0 = tile / p.head_blocks * p.box_rows;
      }
      const int left = j < n ? p.rows - row0 : 0;
      const float* src = p.lse + static_cast<int64_t>(row0) * p.hq + g * p.group + h0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = rr[e] < left && (p.head_blocks == 1 || h0 + (32 * e + lane) % p.box_heads < p.group)
                   ? __ldg(src + at[e]) : INFINITY;
    };
    float v[2][4];
    int b = warp - kWLse;
    uint32_t parity = 1;  // of the stage's use before this one (the first round does not wait)
    fetch(b, v[0]);
    fetch(b + 2, v[1]);
    bool ok = warp_wait(&ctl.k_full, 0, wlim);
    const bool odd_keys = ctl.odd_keys != 0;
    for (int j = b; j < n && ok && !*abort_flag; j += 2) {
      if (j >= kQStages) ok = warp_wait(&ctl.l_empty[b], parity, wlim);
      if (!ok) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // a query whose lse is +inf adds nothing; nor does a column without a query, which needs the bit
        // only where a key makes NaN of its zeros (sums that look at bits take longer)
        const uint32_t bits = __ballot_sync(0xffffffffu, v[0][e] == INFINITY && (odd_keys || 32 * e + lane < columns));
        ctl.lse[b][32 * e + lane] = lse_unit(p, v[0][e]);
        if (lane == 0) ctl.off[b][e] = bits;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.l_full[b]);
      if ((b += 2) >= kQStages) {
        b -= kQStages;
        parity ^= 1;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[0][e] = v[1][e];
      fetch(j + 4, v[1]);
    }
    if (!ok && lane == 0) flag_timeout(p, ctl);
  } else {
    // ------------------------------------------------------------ exponentials and sums
    const int quarter = warp & 3;
    const int t = quarter * 32 + lane, key = key0 + t;
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    // the first sixteen warps: a quarter of key t's row into TMEM (bf16 pairs, the A-operand layout)
    const int part = warp >> 2;
    if (warp < 16) {
      tmem_store(ctl.tmem_base + kKCol + lane_off + part * (D / 8), kreg);
      uint32_t bits = 0;  // bit 15 or 31: an exponent of all ones
#pragma unroll
      for (int c = 0; c < D / 8; ++c) bits |= (kreg[c] & 0x7fff7fffu) + 0x00800080u;
      if (bits & 0x80008000u) ctl.odd_keys = 1;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.k_full);
    }
    const int turn = warp >> 3, half = part & 1;  // tiles turn, turn + 3 ..; queries 64 half ..
    const uint32_t tS = ctl.tmem_base + turn * kTN + 64 * half + lane_off;
    const uint64_t sl2 = f2_pack(p.scale_log2, p.scale_log2);
    float total = 0.f;
    bool ok = true, ready = false;
    int b = turn;  // stage of the tile, and the parity of its use
    uint32_t bp = 0, sp = 0;
    for (int j = turn; j < n; j += kGroups) {
      if (!__all_sync(0xffffffffu, ready)) {
        ok = warp_wait(&ctl.l_full[b], bp, wlim) && warp_wait(&ctl.s_full[turn], sp, wlim);
        if (!ok) break;
      }
      tc_fence_after();
      const float* lse = ctl.lse[b] + 64 * half;
      const uint32_t off0 = ctl.off[b][2 * half], off1 = ctl.off[b][2 * half + 1];
      uint32_t r[32];
      tmem_ld32(tS, r);
      tmem_wait_ld();
      float sum = 0.f;
      if (64 * half < columns) {
        sum = off0 == 0 ? sum32<false>(r, lse, 0, sl2) : sum32<true>(r, lse, off0, sl2);
        if (__any_sync(0xffffffffu, sum > p.large)) sum = exact_sum32<D>(p, sum, g, key, j0 + j, 64 * half);
      }
      tmem_ld32(tS + 32, r);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.s_free[turn]);
      if (64 * half + 32 < columns) {
        float more = off1 == 0 ? sum32<false>(r, lse + 32, 0, sl2) : sum32<true>(r, lse + 32, off1, sl2);
        if (__any_sync(0xffffffffu, more > p.large)) more = exact_sum32<D>(p, more, g, key, j0 + j, 64 * half + 32);
        sum += more;
      }
      // the next tile's stage, and whether it is there (asked ahead)
      const int b_now = b;
      if ((b += kGroups) >= kQStages) {
        b -= kQStages;
        bp ^= 1;
      }
      sp ^= 1;
      ready = j + kGroups < n && mbar_test(&ctl.l_full[b], bp) && mbar_test(&ctl.s_full[turn], sp);
      total += sum;
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.l_empty[b_now]);
    }
    const bool wok = __all_sync(0xffffffffu, ok);
    if (!wok && lane == 0) flag_timeout(p, ctl);
    ctl.red[part][t] = total;
    asm volatile("bar.sync 2, %0;" ::"n"(256 * kGroups) : "memory");  // the groups
    if (part == 0 && wok && key < p.prefix_len) {
      total = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * kGroups; ++k) total += ctl.red[k][t];
      if (p.nsplit > 1)
        p.part[(static_cast<size_t>(blockIdx.x % p.nsplit) * p.hkv + g) * p.prefix_len + key] = total;
      else
        p.w[g * p.w_stride + key] = with_earlier(p, g, key, total);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kWMma) {
    if (lane == 0 && !mbar_wait(&ctl.drained, 0, wlim)) flag_timeout(p, ctl);
    __syncwarp();
    tc_fence_after();
    tmem_dealloc<kTmemCols>(ctl.tmem_base);
  }
}

// ---------------------------------------------------------------- fp32, CUDA cores
// 256 threads (16 x 16) hold 128 keys and take 64 queries at a time through shared memory: thread
// (ty, tx) computes the scores of keys ty + 16 u and queries tx + 16 i (a 16-byte shared-memory
// load serves 4 or 8 dot products), and adds up its keys' exponentials, a tile's four first. What the
// roundings of the sum over the tiles cut off is kept beside it and taken up by the next tile: equal terms, which
// all round the same way, would put a long plain sum off by 7e-5 (73728 terms of a key).
constexpr int kFThreads = 256, kFKeys = 128, kFQueries = 64;

__device__ __forceinline__ int swz(int row, int c) { return c ^ (row & 7); }

template <int D>
constexpr size_t f32_smem() {
  return sizeof(float) * ((kFKeys + 2 * kFQueries) * D + 2 * kFQueries);
}

// (Its registers: with 128 elements one CTA fits on an SM anyway; without the hint a long call takes 7 % more.)
template <int D>
__global__ void __launch_bounds__(kFThreads, D == 128 ? 1 : 0) weights_f32(const __grid_constant__ WeightsParams p) {
  constexpr int kC = D / 4, kU = kFKeys / 16, kI = kFQueries / 16;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  float4* sK = reinterpret_cast<float4*>(smem_raw);
  float4* sQ = sK + kFKeys * kC;  // two tiles
  float* sL = reinterpret_cast<float*>(sQ + 2 * kFQueries * kC);
  grid_dep_launch();
  const int item = blockIdx.x / p.nsplit, part = blockIdx.x % p.nsplit;
  const int g = item / p.key_tiles, key0 = item % p.key_tiles * kFKeys;
  const int j0 = static_cast<int>(static_cast<long long>(p.q_tiles) * part / p.nsplit);
  const int j1 = static_cast<int>(static_cast<long long>(p.q_tiles) * (part + 1) / p.nsplit);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int64_t queries = static_cast<int64_t>(p.rows) * p.group;
  for (int i = tid; i < kFKeys * kC; i += kFThreads) {
    const int r = i / kC, c = i % kC;
    const bool in = key0 + r < p.prefix_len;
    cp_async16(sK + r * kC + swz(r, c),
               static_cast<const float*>(p.pk) +
                   (in ? (key0 + r) * p.row_stride + g * p.head_stride + 4 * c : 0), in ? 16 : 0);
  }
  auto load = [&](int j, int b) {
    for (int i = tid; i < kFQueries * kC; i += kFThreads) {
      const int t = i / kC, c = i % kC;
      const int64_t m = static_cast<int64_t>(j) * kFQueries + t;
      const bool in = m < queries;
      const int64_t at = in ? m / p.group * p.hq + g * p.group + m % p.group : 0;
      cp_async16(sQ + (b * kFQueries + t) * kC + swz(t, c), static_cast<const float*>(p.q) + at * D + 4 * c,
                 in ? 16 : 0);
    }
    cp_async_commit();
    if (tid < kFQueries) {
      const int64_t m = static_cast<int64_t>(j) * kFQueries + tid;
      sL[b * kFQueries + tid] = lse_unit(
          p, m < queries ? __ldg(p.lse + m / p.group * p.hq + g * p.group + m % p.group) : INFINITY);
    }
  };
  load(j0, 0);
  float total[kU], over[kU];  // the sum, and what its last rounding added to it
#pragma unroll
  for (int u = 0; u < kU; ++u) total[u] = over[u] = 0.f;
  for (int j = j0; j < j1; ++j) {
    const int b = (j - j0) & 1;
    cp_async_wait_all();
    __syncthreads();  // tile j is there, and tile j - 1 has been read
    if (j + 1 < j1) load(j + 1, b ^ 1);
    const float4* q = sQ + b * kFQueries * kC;
    float s[kU][kI];
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int i = 0; i < kI; ++i) s[u][i] = 0.f;
#pragma unroll 4
    for (int c = 0; c < kC; ++c) {
      float4 qf[kI];
#pragma unroll
      for (int i = 0; i < kI; ++i) qf[i] = q[(tx + 16 * i) * kC + swz(tx, c)];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const float4 kf = sK[(ty + 16 * u) * kC + swz(ty, c)];
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          s[u][i] = fmaf(qf[i].x, kf.x, s[u][i]);
          s[u][i] = fmaf(qf[i].y, kf.y, s[u][i]);
          s[u][i] = fmaf(qf[i].z, kf.z, s[u][i]);
          s[u][i] = fmaf(qf[i].w, kf.w, s[u][i]);
        }
      }
    }
    float sum[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) sum[u] = -over[u];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const float lse = sL[b * kFQueries + tx + 16 * i];
      if (lse == -INFINITY) continue;  // adds nothing, whatever q holds
#pragma unroll
      for (int u = 0; u < kU; ++u) sum[u] += exp2f(fmaf(s[u][i], p.scale_log2, lse));
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const float to = total[u] + sum[u];
      over[u] = (to - total[u]) - sum[u];
      if (!(fabsf(over[u]) < INFINITY)) over[u] = 0.f;  // (an infinite sum stays one)
      total[u] = to;
    }
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    float sum = total[u];
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    const int key = key0 + ty + 16 * u;
    if (tx != 0 || key >= p.prefix_len) continue;
    if (p.nsplit > 1)
      p.part[(static_cast<size_t>(part) * p.hkv + g) * p.prefix_len + key] = sum;
    else
      p.w[g * p.w_stride + key] = with_earlier(p, g, key, sum);
  }
}

// The parts of a split launch, added in order; without parts (no rows) what is left of the earlier
// sum.
__global__ void __launch_bounds__(256) weights_join(const __grid_constant__ WeightsParams p) {
  grid_dep_wait();
  const int key = static_cast<int>(blockIdx.x * 256u + threadIdx.x);
  const int g = blockIdx.y;
  if (key >= p.prefix_len) return;
  float sum = 0.f;
#pragma unroll 8
  for (int c = 0; c < p.nsplit; ++c)
    sum += p.part[(static_cast<size_t>(c) * p.hkv + g) * p.prefix_len + key];
  p.w[g * p.w_stride + key] = with_earlier(p, g, key, sum);
}

// ---------------------------------------------------------------- host side
constexpr int kParts = 64;               // parts of a split launch at most
constexpr long long kSplitCtas = 2048;   // CTAs of a split launch at most

template <int D>
cudaError_t launch_tc(const WeightsParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap q;
  if (!make_map3(&q, p.q, D, p.hq, p.rows, D, static_cast<int64_t>(p.hq) * D, p.box_heads, p.box_rows))
    return cudaErrorInvalidValue;
  const cudaError_t e = ensure_smem_attr(weights_tc<D>, smem_bytes<D>(), done);
  if (e != cudaSuccess) return e;
  const AttnLaunch L(static_cast<unsigned>(p.hkv) * p.key_tiles * p.nsplit, kThreads, smem_bytes<D>(),
                     stream, 1, false);
  return cudaLaunchKernelEx(&L.cfg, weights_tc<D>, p, q);
}

template <int D>
cudaError_t launch_f32(const WeightsParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = ensure_smem_attr(weights_f32<D>, f32_smem<D>(), done);
  if (e != cudaSuccess) return e;
  const AttnLaunch L(static_cast<unsigned>(p.hkv) * p.key_tiles * p.nsplit, kFThreads, f32_smem<D>(),
                     stream, 1, false);
  return cudaLaunchKernelEx(&L.cfg, weights_f32<D>, p);
}

// Whether [hkv, len] elements at a and at b, rows sa and sb apart, may have one in common: with one
// stride exactly, otherwise by the first and the last.
bool share(const float* a, int64_t sa, const float* b, int64_t sb, int64_t len, int hkv) {
  const int64_t at = (reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a)) / 4;
  if (at >= (hkv - 1) * sa + len || -at >= (hkv - 1) * sb + len) return false;
  const int64_t off = sa == sb ? (at % sa + sa) % sa : 0;  // of b's rows behind a's
  return off < len || off > sa - len;
}

dard_status prepare(const dard_prefix_weights_args* a, WeightsParams& p) {
  memset(&p, 0, sizeof(p));
  if (!a) return report(DARD_ERR_NULL, "args is NULL");
  if (a->dtype != DARD_BF16 && a->dtype != DARD_F32)
    return report(DARD_ERR_VALUE, "dtype %d is neither DARD_F32 nor DARD_BF16", a->dtype);
  if (a->rows < 0) return report(DARD_ERR_SHAPE, "rows %d < 0", a->rows);
  if (a->hq < 1 || a->hkv < 1 || a->hq % a->hkv != 0)
    return report(DARD_ERR_SHAPE, "hq %d / hkv %d: need hq %% hkv == 0", a->hq, a->hkv);
  if (a->hkv > 65535) return report(DARD_ERR_SHAPE, "hkv %d above 65535", a->hkv);
  if (a->head_dim != 64 && a->head_dim != 128)
    return report(DARD_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", a->head_dim);
  if (a->prefix_len < 0 || a->prefix_len > DARD_PREFIX_MAX_LEN)
    return report(DARD_ERR_SHAPE, "prefix_len %d outside 0..%d", a->prefix_len, DARD_PREFIX_MAX_LEN);
  if (!(a->scale >= 0.f) || !std::isfinite(a->scale))
    return report(DARD_ERR_VALUE, "scale must be finite and >= 0");
  if (!std::isfinite(a->decay)) return report(DARD_ERR_VALUE, "decay must be finite");
  if (a->prefix_len == 0) return DARD_OK;
  if (!a->weights) return report(DARD_ERR_NULL, "weights is NULL");
  if (a->weights_stride < a->prefix_len || (a->weights_in && a->weights_in_stride < a->prefix_len))
    return report(DARD_ERR_SHAPE, "a weights stride is below prefix_len");
  if (a->weights_in == a->weights && a->weights_in_stride != a->weights_stride)
    return report(DARD_ERR_VALUE, "weights_in may be weights with the same stride only");
  if (a->weights_in && a->weights_in != a->weights &&
      share(a->weights, a->weights_stride, a->weights_in, a->weights_in_stride, a->prefix_len, a->hkv))
    return report(DARD_ERR_VALUE, "weights_in must be weights or lie apart from it");
  if (((reinterpret_cast<uintptr_t>(a->weights) | reinterpret_cast<uintptr_t>(a->weights_in) |
        reinterpret_cast<uintptr_t>(a->lse)) & 3u) != 0)
    return report(DARD_ERR_ALIGN, "weights, weights_in and lse must be 4-byte aligned");
  const int esz = a->dtype == DARD_BF16 ? 2 : 4;
  if (a->rows > 0) {
    if (!a->q || !a->lse || !a->prefix_k) return report(DARD_ERR_NULL, "q, lse or prefix_k is NULL");
    if (static_cast<long long>(a->rows) * a->hq > (1ll << 31) - 256)
      return report(DARD_ERR_SHAPE, "rows times hq exceed 2^31 - 256");
    if (a->prefix_row_stride < a->head_dim || a->prefix_head_stride < a->head_dim ||
        a->prefix_row_stride > (1ll << 36) || a->prefix_head_stride > (1ll << 36))
      return report(DARD_ERR_SHAPE, "prefix strides outside head_dim..2^36");
    if (((reinterpret_cast<uintptr_t>(a->q) | reinterpret_cast<uintptr_t>(a->prefix_k) |
          static_cast<uintptr_t>(a->prefix_row_stride * esz) |
          static_cast<uintptr_t>(a->prefix_head_stride * esz)) & 15u) != 0)
      return report(DARD_ERR_ALIGN, "q, prefix_k and its strides must be multiples of 16 bytes");
  }
  const size_t need = dard_prefix_weights_workspace_size(a->rows, a->hq, a->hkv, a->head_dim,
                                                         a->prefix_len);
  if (a->workspace && a->workspace_bytes < need)
    return report(DARD_ERR_WORKSPACE, "workspace of %zu bytes needed", need);
  if ((reinterpret_cast<uintptr_t>(a->workspace) & 15u) != 0)
    return report(DARD_ERR_ALIGN, "workspace must be 16-byte aligned");
  p.q = a->q;
  p.lse = a->lse;
  p.pk = a->prefix_k;
  p.w_in = a->weights_in;
  p.w = a->weights;
  p.part = static_cast<float*>(a->workspace);
  p.status = a->status;
  p.row_stride = a->prefix_row_stride;
  p.head_stride = a->prefix_head_stride;
  p.w_in_stride = a->weights_in_stride;
  p.w_stride = a->weights_stride;
  p.rows = a->rows;
  p.hq = a->hq;
  p.hkv = a->hkv;
  p.prefix_len = a->prefix_len;
  p.group = a->hq / a->hkv;
  p.decay = a->decay;
  p.scale_log2 = (a->scale > 0.f ? a->scale : 1.0f / std::sqrt(static_cast<float>(a->head_dim))) * kLog2e;
  p.scale = (a->scale > 0.f ? static_cast<double>(a->scale) : 1.0 / std::sqrt(static_cast<double>(a->head_dim))) *
            1.4426950408889634;
  // lse in the unit in which scale_log2, rounded to 32 bits, takes the scores: its rounding then counts for their
  // difference only. (Scores from the tensor cores come short, as a running sum is cut: weights of random q and k
  // of 128 elements by some 1e-7 of themselves. Nothing makes up for that: how much it is depends on the keys.)
  const double unit = p.scale_log2 / p.scale * 1.4426950408889634;
  p.lse_hi = static_cast<float>(-unit);
  p.lse_lo = static_cast<float>(-unit - p.lse_hi);
  p.test_drop_kv = -1;
  return DARD_OK;
}

// Parts of the split, by the time of a launch in query tiles: a CTA costs `start` beside its tiles, the
// join `join`; a launch with no more CTAs than SMs takes its longest, a larger one total / SMs plus half
// a CTA. Bounded by what the workspace holds.
int choose_parts(long long items, int q_tiles, int sms, double start, double join) {
  long long best = 1;
  double best_time = 0;
  for (long long s = 1; s <= std::min<long long>(kParts, q_tiles) && (s == 1 || items * s <= kSplitCtas); ++s) {
    const double cta = start + std::ceil(static_cast<double>(q_tiles) / s);
    const double n = static_cast<double>(items) * s;
    const double time = (n <= sms ? cta : n * (start + static_cast<double>(q_tiles) / s) / sms + 0.5 * cta) +
                        (s > 1 ? join : 0.0);
    if (s == 1 || time < best_time) {
      best = s;
      best_time = time;
    }
  }
  return static_cast<int>(best);
}

}  // namespace
}  // namespace dard

extern "C" {

size_t dard_prefix_weights_workspace_size(int32_t rows, int32_t hq, int32_t hkv, int32_t head_dim,
                                          int32_t prefix_len) {
  using namespace dard;
  if (rows < 0 || hq < 1 || hkv < 1 || hq % hkv != 0 || (head_dim != 64 && head_dim != 128) ||
      prefix_len < 0 || prefix_len > DARD_PREFIX_MAX_LEN)
    return 0;
  // at most kSplitCtas CTAs of 128 keys, so that many parts of 128 sums each
  return kSplitCtas * 128 * sizeof(float);
}

dard_status dard_prefix_weights(const dard_prefix_weights_args* args, void* stream_ptr) {
  using namespace dard;
  report(DARD_OK, "%s", "");
  WeightsParams p;
  const dard_status st = prepare(args, p);
  if (st != DARD_OK) return st;
  if (args->prefix_len == 0) return DARD_OK;
  const cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
  if (const char* w = std::getenv("DARD_TEST_WAIT_CYCLES")) p.wait_cycles = std::atoll(w);
  if (const char* d = std::getenv("DARD_TEST_DROP_KV")) p.test_drop_kv = std::atoi(d);
  if (std::getenv("DARD_TEST_FAIL_LAUNCH") != nullptr)
    return report(DARD_ERR_CUDA, "prefix weights launch failed: %s (DARD_TEST_FAIL_LAUNCH)",
                  cudaGetErrorString(cudaErrorLaunchFailure));
  const bool bf16 = args->dtype == DARD_BF16;
  cudaError_t e = cudaSuccess;
  if (p.rows > 0) {
    p.key_tiles = (p.prefix_len + 127) / 128;
    if (bf16) {
      p.box_heads = std::min(p.group, 128);
      p.box_rows = std::min(128 / p.box_heads, p.rows);
      p.head_blocks = (p.group + p.box_heads - 1) / p.box_heads;
      p.q_tiles = (p.rows + p.box_rows - 1) / p.box_rows * p.head_blocks;
      p.large = 0.25f * std::min(32, p.box_rows * p.box_heads);
    } else {
      p.q_tiles = static_cast<int32_t>((static_cast<long long>(p.rows) * p.group + kFQueries - 1) / kFQueries);
    }
    const long long items = static_cast<long long>(p.key_tiles) * p.hkv;
    if (items > (1ll << 31) - 1) return report(DARD_ERR_SHAPE, "too many key tiles");
    p.nsplit = !p.part ? 1 : bf16 ? choose_parts(items, p.q_tiles, sm_count(), 10.0, 8.0)
                                  : choose_parts(items, p.q_tiles, sm_count(), 1.5, 1.0);
    if (!bf16)
      e = args->head_dim == 64 ? launch_f32<64>(p, stream) : launch_f32<128>(p, stream);
    else
      e = args->head_dim == 64 ? launch_tc<64>(p, stream) : launch_tc<128>(p, stream);
  }
  if (e == cudaSuccess && p.nsplit != 1) {
    AttnLaunch L((p.prefix_len + 255) / 256, 256, 0, stream, 1, p.nsplit > 1);
    L.cfg.gridDim.y = p.hkv;
    e = cudaLaunchKernelEx(&L.cfg, weights_join, p);
  }
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "prefix weights launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
