// dard_prefix_attn.cu - attention of a decoding step over a prefix that the batch shares and each
// sequence's own rows (dard_prefix_attention): validation, the split of the keys, the bf16 kernel
// on the tensor cores and the kernel that joins the parts of a split.
//
// prefix_tc: 128 packed queries (dard_prefix.cuh) of one key/value head against a run of key
// tiles of 128: first the prefix's, with no mask but the ragged end of the last, then the rows of
// the sequences that the tile touches, under each row's mask. One pass with a running maximum and
// sum (the probabilities never leave the chip), fp32 accumulators. 20 warps:
//   warps 0-15 softmax and epilogue: warps q, q + 4, q + 8 and q + 12 share TMEM lane quarter q
//              (queries 32q .. 32q + 31), each taking 32 of a tile's 128 keys;
//   warp 16    TMA producer of K, through 3 stages;
//   warp 17    TMEM allocator and PV issuer: O += P_j V_j, P_j (bf16) read from TMEM;
//   warp 18    S issuer: S_j = Q K_j^T (Q from TMEM, K from shared memory) into a ring of two
//              128-column TMEM buffers;
//   warp 19    TMA producer of V, through 3 stages (K runs ahead of V by two tiles: one producer of
//              both would hold K up for V's stages).
// TMEM: S ring [0, 256), O [256, 256 + D), P [384, 448), Q [448, 448 + D/2).
// Bound by the chain of one tile's softmax (load, maximum over four warps, exponentials, hand-over):
// about 1570 cycles per 128 x 128 scores, of which the tensor cores work 1024 and the special-function units
// 500. Measured: 4608 rows of 28 heads on 4 of 128 over 32768 keys 1.54-1.63 ms (1340-1420 TFLOP/s); one token
// over 4096 keys 8.8-9.8 us with its join. Sixteen softmax warps instead of eight: 1732 -> 1571 us when they
// came in.
//
// Values that are not finite: the product with V multiplies every key of a tile by every query's
// weight, and 0 times NaN is NaN. Keys of the prefix are seen by every query (rows behind its end
// arrive as zeros), but an own tile holds copies and sequences that a query does not see. The
// softmax warps look through an own tile's V, a sixteenth each, before they hand their weights over:
// such values are taken out of V before the product and added to the queries that do see the key.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "dard_prefix.cuh"

namespace dard {
namespace {

constexpr int kThreads = 640;
constexpr int kNS = 2;   // S buffers in TMEM
constexpr int kNKV = 3;  // TMA stages for K and for V
constexpr int kSoftmaxWarps = 16;
constexpr int kParts = 4;              // warps that share a query's keys
constexpr int kCols = kTN / kParts;    // keys of a tile per thread
constexpr int kWK = 16, kWPV = 17, kWS = 18, kWV = 19;

// Every barrier completes one phase per use of its ring slot; tile j uses slot j % ring and waits
// for parity (j / ring) & 1. Each wait for use u of a slot is preceded, in the same thread or
// through a chain of waits, by the completion of use u - 1 (the parity would alias otherwise).
struct __align__(16) Ctl {
  uint64_t q_full, o_full, p_full, pv_done;
  uint64_t k_full[kNKV], k_empty[kNKV], v_full[kNKV], v_empty[kNKV];
  uint64_t s_full[kNS], s_free[kNS];
  uint64_t drained;       // every product both issuers launched has completed (two commits)
  uint32_t tmem_base;
  int32_t abort;
  int32_t poison;         // a query sees a value that is not finite
  float red_max[2][kParts][kBM];  // per tile parity: the column parts' row maxima
  float red_sum[2][kParts][kBM];  // their row sums: of the weights, of the weights rounded to bf16
  int64_t out_row[kBM];      // packed query -> row * hq + head, or -1 (not stored)
  RowMasks row_mask[kBM];
  BlockScratch scratch[4];
  int32_t row_seq[kBM];      // -1: no query
  uint32_t inf_pos[kBM][4], inf_neg[kBM][4];  // elements to become inf, -inf (both: NaN)
};

template <int D>
constexpr size_t smem_bytes() {
  return 1024 + 2 * kNKV * static_cast<size_t>(kTN) * D * 2 + sizeof(Ctl);
}

__device__ __forceinline__ void flag_timeout(const PrefixParams& p, Ctl& ctl) {
  ctl.abort = 1;
  if (p.a.status) atomicOr(p.a.status, DARD_STATUS_TIMEOUT);
}

// A sixteenth (`share`) of an own tile of V in shared memory: values that are not finite become
// zeros, and the queries that see their keys are marked. `row0` is the tile's first row of k and v.
// Called by whole warps, after row_mask and row_seq are written.
template <int D>
__device__ __forceinline__ void check_values(const PrefixParams& p, Ctl& ctl, uint8_t* tile, int row0,
                                             int share) {
  constexpr int kChunks = kTN * D / 8 / kSoftmaxWarps;  // 16-byte chunks of the warp
  const int lane = threadIdx.x & 31;
  uint32_t bits = 0;  // bit 15 or 31: an exponent of all ones
#pragma unroll
  for (int u = 0; u < kChunks / 32; ++u) {
    const uint4 x = *reinterpret_cast<const uint4*>(tile + 16 * (share * kChunks + 32 * u + lane));
    bits |= ((x.x & 0x7fff7fffu) + 0x00800080u) | ((x.y & 0x7fff7fffu) + 0x00800080u) |
            ((x.z & 0x7fff7fffu) + 0x00800080u) | ((x.w & 0x7fff7fffu) + 0x00800080u);
  }
  if (!__any_sync(0xffffffffu, bits & 0x80008000u)) return;
  for (int u = 0; u < kChunks / 32; ++u) {
    const int i = share * kChunks + 32 * u + lane;
    uint16_t* v = reinterpret_cast<uint16_t*>(tile + 16 * i);
    const int key = (i >> 3) % kTN;
    const int e0 = (i >> 3) / kTN * 64 + (((i & 7) ^ (key & 7)) << 3);
    uint32_t pos = 0, neg = 0;  // of the chunk's 8 elements
    for (int e = 0; e < 8; ++e) {
      const uint32_t b = v[e];
      if ((b & 0x7f80u) != 0x7f80u) continue;
      if ((b & 0x7fu) || !(b & 0x8000u)) pos |= 1u << e;
      if ((b & 0x7fu) || (b & 0x8000u)) neg |= 1u << e;
      v[e] = 0;
    }
    if (!(pos | neg)) continue;
    for (int t = 0; t < kBM; ++t) {
      const int s = ctl.row_seq[t];
      if (s < 0 || !(own_vis64(p.a.seq[s], row0 + key - p.a.seq[s].row_base, ctl.row_mask[t]) & 1))
        continue;
      if (pos) atomicOr(&ctl.inf_pos[t][e0 >> 5], pos << (e0 & 31));
      if (neg) atomicOr(&ctl.inf_neg[t][e0 >> 5], neg << (e0 & 31));
      ctl.poison = 1;
    }
  }
  fence_proxy_async_smem();  // the zeros, before the product reads the tile
  __syncwarp();
}

__device__ __forceinline__ float poisoned(const Ctl& ctl, int t, int e, float o) {
  const bool pos = ctl.inf_pos[t][e >> 5] >> (e & 31) & 1, neg = ctl.inf_neg[t][e >> 5] >> (e & 31) & 1;
  if (pos) o += INFINITY;
  if (neg) o -= INFINITY;
  return o;
}

// All softmax threads, and those of the four warps of TMEM lane quarter q.
__device__ __forceinline__ void all_bar_sync() {
  asm volatile("bar.sync 2, 512;" ::: "memory");
}
__device__ __forceinline__ void quarter_bar_sync(int q) {
  asm volatile("bar.sync %0, 128;" ::"r"(3 + q) : "memory");
}
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    prefix_tc(const __grid_constant__ PrefixParams p, const __grid_constant__ CUtensorMap tpk,
              const __grid_constant__ CUtensorMap tpv, const __grid_constant__ CUtensorMap tk,
              const __grid_constant__ CUtensorMap tv) {
  constexpr int kSub = D / 64;                 // 128-byte (64 x bf16) column blocks
  constexpr uint32_t kKSub = kTN * 128;        // one 128-row x 128-byte swizzled block
  constexpr uint32_t kKVBytes = kSub * kKSub;  // one K (or V) tile of 128 keys
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* sK = base;                  // kNKV stages
  uint8_t* sV = sK + kNKV * kKVBytes;  // kNKV stages
  Ctl& ctl = *reinterpret_cast<Ctl*>(sV + kNKV * kKVBytes);

  grid_dep_launch();  // the launch that joins the parts may be scheduled; it waits for this one
  // (The work's bounds come before any branch on the warp: behind one the compiler holds them per
  // thread, and the loops below run 6 % slower.)
  const int item = blockIdx.x / p.nsplit, part = blockIdx.x % p.nsplit;
  const int g = item / p.tiles, m0 = item % p.tiles * kBM;
  int s0, s1, key0, key_end;
  own_range(p, item % p.tiles, kBM, s0, s1, key0, key_end);
  const int npt = (p.prefix_len + kTN - 1) / kTN;  // the prefix's tiles
  const int all = npt + (key_end - key0 + kTN - 1) / kTN;
  const int j0 = static_cast<int>(static_cast<long long>(all) * part / p.nsplit);
  const int n_kt = static_cast<int>(static_cast<long long>(all) * (part + 1) / p.nsplit) - j0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long wlim = p.a.wait_cycles > 0 ? p.a.wait_cycles : kWaitCycles;
  const int first_own = max(npt - j0, 0);  // local index of the first own tile (may be >= n_kt)

  auto load_kv = [&](int j, bool k_or_v) {
    const int b = j % kNKV;
    uint64_t* bar = k_or_v ? &ctl.k_full[b] : &ctl.v_full[b];
    uint8_t* dst = (k_or_v ? sK : sV) + b * kKVBytes;
    const bool own = j >= first_own;
    const void* map = k_or_v ? (own ? &tk : &tpk) : (own ? &tv : &tpv);
    const int row = own ? key0 + (j0 + j - npt) * kTN : (j0 + j) * kTN;
    mbar_arrive_expect_tx(bar, kKVBytes);
    if (k_or_v && j == p.a.test_drop_kv) return;  // test hook: this K copy is never issued
#pragma unroll
    for (int s = 0; s < kSub; ++s) tma_load_3d(dst + s * kKSub, map, bar, s * 64, row, g);
  };
  if (warp == kWK && lane == 0) {
    mbar_init(&ctl.q_full, kSoftmaxWarps);
    mbar_init(&ctl.drained, 2);
    mbar_init(&ctl.o_full, 1);
    mbar_init(&ctl.p_full, kSoftmaxWarps);
    mbar_init(&ctl.pv_done, 1);
    for (int b = 0; b < kNKV; ++b) {
      mbar_init(&ctl.k_full[b], 1);
      mbar_init(&ctl.k_empty[b], 1);
      mbar_init(&ctl.v_full[b], 1);
      mbar_init(&ctl.v_empty[b], 1);
    }
    for (int b = 0; b < kNS; ++b) {
      mbar_init(&ctl.s_full[b], 1);
      mbar_init(&ctl.s_free[b], kSoftmaxWarps);
    }
    ctl.abort = 0;
    ctl.poison = 0;
    fence_barrier_init();
    load_kv(0, true);  // (the rest follows behind the block's barrier)
    load_kv(0, false);
  }
  if (warp == kWPV) {
    tmem_alloc<kTmemCols>(&ctl.tmem_base);
    tmem_relinquish();
  }
  // Softmax warp w: queries 32 (w % 4) .. + 31 (TMEM lane quarter), keys 32 (w / 4) .. of a tile
  const int quarter = warp & 3, part4 = warp >> 2;
  const int t = quarter * 32 + lane;  // this thread's query within the tile
  constexpr int kOC = D / kParts;     // its share of the output's columns
  uint32_t qreg[D / 8];               // a quarter of its row of q
  int seq = -1, r = 0;                // its sequence and sequence-relative row
  int64_t out_row = -1;
  if (warp < kSoftmaxWarps) {
    if (m0 + t < p.queries) {
      const int tq = (m0 + t) / p.group;
      seq = seq_of_query(p, tq, s0, s1 + 1);
      r = p.a.seq[seq].q_start + tq - p.q_before[seq];
      out_row = static_cast<int64_t>(p.a.seq[seq].row_base + r) * p.a.hq + g * p.group +
                (m0 + t) % p.group;
    }
    const uint4* src = reinterpret_cast<const uint4*>(
        static_cast<const __nv_bfloat16*>(p.a.q) + out_row * D + part4 * kOC);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const uint4 u = seq >= 0 ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
      qreg[4 * c] = u.x;
      qreg[4 * c + 1] = u.y;
      qreg[4 * c + 2] = u.z;
      qreg[4 * c + 3] = u.w;
    }
    if (part4 == 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) ctl.inf_pos[t][e] = ctl.inf_neg[t][e] = 0;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tO = ctl.tmem_base + kNS * kTN;
  const uint32_t tP = ctl.tmem_base + 384;
  const uint32_t tQ = ctl.tmem_base + 448;
  volatile int32_t* abort_flag = &ctl.abort;

  if (warp == kWK || warp == kWV) {
    // ------------------------------------------------------------ TMA producers
    if (lane == 0) {
      const bool is_k = warp == kWK;
      uint64_t* full = is_k ? ctl.k_full : ctl.v_full;
      uint64_t* empty = is_k ? ctl.k_empty : ctl.v_empty;
      int last = 0;
      for (int j = 1; j < n_kt && !*abort_flag; ++j) {
        if (j >= kNKV && !mbar_wait(&empty[j % kNKV], ((j - kNKV) / kNKV) & 1, wlim)) {
          flag_timeout(p, ctl);
          break;
        }
        load_kv(j, is_k);
        last = j;
      }
      // Every copy issued lands before shared memory is released: the latest use of each stage.
      for (int b = 0; b < kNKV; ++b) {
        const int jb = last - ((last - b) % kNKV + kNKV) % kNKV;
        if (jb >= 0 && !(is_k && jb == p.a.test_drop_kv)) mbar_wait(&full[b], (jb / kNKV) & 1, wlim);
      }
    }
  } else if (warp == kWS) {
    // ------------------------------------------------------------ S issuer
    // (both issuers: the whole warp walks the loop, so that what it computes is uniform over the
    // warp and stays in uniform registers; one elected lane issues)
    constexpr uint32_t kIdS = idesc_bf16_f32(kBM, kTN, 0, 0);
    const bool issue = elect_one();
    const uint64_t desc = smem_desc_sw128(smem_u32(sK), 16, 1024);
    bool ok = warp_wait(&ctl.q_full, 0, wlim);
    for (int j = 0; j < n_kt && ok; ++j) {
      const int kb = j % kNKV, sb = j % kNS;
      if (j >= kNS) ok = warp_wait(&ctl.s_free[sb], ((j - kNS) / kNS) & 1, wlim);
      ok = ok && warp_wait(&ctl.k_full[kb], (j / kNKV) & 1, wlim);
      if (!ok) break;
      tc_fence_after();
      if (issue) {
        const uint64_t dk = desc + kb * (kKVBytes / 16);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          mma_ts(ctl.tmem_base + sb * kTN, tQ + ks * 8, dk + (ks >> 2) * (kKSub / 16) + (ks & 3) * 2, kIdS, ks > 0);
        mma_commit(&ctl.s_full[sb]);
        mma_commit(&ctl.k_empty[kb]);
      }
    }
    if (!ok && lane == 0) flag_timeout(p, ctl);
    if (issue) mma_commit(&ctl.drained);
    __syncwarp();
  } else if (warp == kWPV) {
    // ------------------------------------------------------------ PV issuer
    constexpr uint32_t kIdO = idesc_bf16_f32(kBM, D, 0, 1);
    const bool issue = elect_one();
    const uint64_t desc = smem_desc_sw128(smem_u32(sV), kKSub, 1024);
    bool ok = true;
    for (int j = 0; j < n_kt && ok; ++j) {
      const int vb = j % kNKV;
      ok = warp_wait(&ctl.v_full[vb], (j / kNKV) & 1, wlim) && warp_wait(&ctl.p_full, j & 1, wlim);
      if (!ok) break;
      tc_fence_after();
      if (issue) {
        const uint64_t dv = desc + vb * (kKVBytes / 16);
#pragma unroll
        for (int ks = 0; ks < kTN / 16; ++ks)
          mma_ts(tO, tP + ks * 8, dv + ks * (2048 / 16), kIdO, (j > 0 || ks > 0) ? 1u : 0u);
        mma_commit(&ctl.pv_done);
        mma_commit(&ctl.v_empty[vb]);
        if (j == n_kt - 1) mma_commit(&ctl.o_full);
      }
    }
    if (!ok && lane == 0) flag_timeout(p, ctl);
    if (issue) mma_commit(&ctl.drained);
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax + epilogue
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    // this warp's quarter of the query rows into TMEM (bf16 pairs, the A-operand layout)
    tmem_store(tQ + lane_off + part4 * (D / 8), qreg);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl.q_full);
    // the last part holds the sequences' last rows: it always has own tiles, and it alone decides
    // which rows are stored
    int store = seq >= 0;
    if (first_own < n_kt) {
      if (part4 == 0) {
        ctl.row_mask[t] = warp_query_masks(p.a, ctl.scratch[quarter], seq, r, g == 0, store);
        ctl.row_seq[t] = seq;
        ctl.out_row[t] = store ? out_row : -1;
      }
      all_bar_sync();  // (check_values() reads every row's mask)
    } else if (part4 == 0) {
      ctl.out_row[t] = out_row;
    }
    const float sl = p.a.scale_log2;
    float m_run = -INFINITY, l_run = 0.f, l_rnd = 0.f;
    // from here on tiles have keys that some query does not see
    const int first_masked = min(first_own, p.prefix_len / kTN - j0);
    bool ok = true, ready = false;
    int missed = 0;  // tiles whose barrier this warp has not come to
    for (int j = 0; j < n_kt; ++j) {
      const int b = j & (kNS - 1);
      // (A warp whose wait runs out leaves, hands nothing over any more and catches up on the barriers behind the
      // loop.)
      if (!__all_sync(0xffffffffu, ready)) {
        ok = warp_wait(&ctl.s_full[b], (j / kNS) & 1, wlim);
        if (!ok) {
          missed = n_kt - j;
          break;
        }
      }
      tc_fence_after();
      uint32_t s[kCols];
      tmem_load(ctl.tmem_base + b * kTN + kCols * part4 + lane_off, s);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.s_free[b]);
      if (j >= first_masked) {
        uint32_t vis = 0;
        if (j < first_own)
          vis = static_cast<uint32_t>(first64(p.prefix_len - (j0 + j) * kTN - kCols * part4));
        else if (seq >= 0)
          vis = static_cast<uint32_t>(own_vis64(
              p.a.seq[seq], key0 + (j0 + j - npt) * kTN + kCols * part4 - p.a.seq[seq].row_base,
              ctl.row_mask[t]));
#pragma unroll
        for (int k = 0; k < kCols; ++k) s[k] = (vis >> k) & 1u ? s[k] : 0xff800000u;  // -inf
      }
      float mx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        mx[e] = fmax3(__uint_as_float(s[e]), __uint_as_float(s[8 + e]), __uint_as_float(s[16 + e]));
#pragma unroll
      for (int e = 0; e < 4; ++e)
        mx[e] = fmax3(mx[e], __uint_as_float(s[24 + e]), fmaxf(mx[4 + e], __uint_as_float(s[28 + e])));
      ctl.red_max[j & 1][part4][t] = fmaxf(fmax3(mx[0], mx[1], mx[2]), mx[3]);
      quarter_bar_sync(quarter);
      const float* red = &ctl.red_max[j & 1][0][t];
      const float mt = fmaxf(fmax3(red[0], red[kBM], red[2 * kBM]), red[3 * kBM]);
      // The reference maximum rises on the first finite value, or when the tile's exceeds it by
      // more than 2^kRescaleLog2 in probability; only then is O rescaled. The warps of a row take
      // the same decision from the same values.
      float m_new = m_run;
      if (m_run == -INFINITY) m_new = mt;
      else if ((mt - m_run) * sl > kRescaleLog2) m_new = mt;
      const bool rescale = (m_new != m_run) && (m_run != -INFINITY);
      const float alpha = rescale ? ex2_approx((m_run - m_new) * sl) : 1.f;
      const float mL = (m_new == -INFINITY) ? 0.f : m_new * sl;
      const bool pv_done = j == 0 || mbar_test(&ctl.pv_done, (j - 1) & 1);  // (asked ahead)
      uint32_t pk[kCols / 2];
      const uint64_t sl2 = f2_pack(sl, sl), nmL2 = f2_pack(-mL, -mL);
      uint64_t acc[2] = {0, 0};  // bit pattern 0 = +0.0f
#pragma unroll
      for (int e = 0; e < kCols / 2; ++e) {
        float x0, x1;
        f2_unpack(f2_fma(f2_pack(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), sl2, nmL2), x0, x1);
        x0 = ex2_approx(x0);
        x1 = ex2_approx(x1);
        pk[e] = pack_bf16x2(x0, x1);
        acc[e & 1] = f2_add(acc[e & 1], f2_pack(x0, x1));
      }
      // P_j replaces P_{j-1}, and O may be rescaled, once PV_{j-1} has completed
      if (!__all_sync(0xffffffffu, pv_done)) {
        ok = warp_wait(&ctl.pv_done, (j - 1) & 1, wlim);
        if (!ok) {
          missed = n_kt - j - 1;
          break;
        }
      }
      tc_fence_after();
      if (__any_sync(0xffffffffu, rescale)) {  // this warp's share of the O columns
        uint32_t rr[kOC];
        tmem_load(tO + lane_off + part4 * kOC, rr);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < kOC; ++e) rr[e] = __float_as_uint(__uint_as_float(rr[e]) * alpha);
        tmem_store(tO + lane_off + part4 * kOC, rr);
      }
      tmem_store(tP + lane_off + part4 * (kCols / 2), pk);
      if (j >= first_own) {
        // (the stage's use before this one has landed: PV_{j-1} has completed, and this use ends
        // only after this warp's weights)
        ok = mbar_wait(&ctl.v_full[j % kNKV], (j / kNKV) & 1, wlim);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          missed = n_kt - j - 1;
          break;
        }
        check_values<D>(p, ctl, sV + j % kNKV * kKVBytes, key0 + (j0 + j - npt) * kTN, warp);
      }
      ready = j + 1 < n_kt && mbar_test(&ctl.s_full[(j + 1) & (kNS - 1)], ((j + 1) / kNS) & 1);  // (asked ahead)
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.p_full);
      float a0, a1;
      f2_unpack(f2_add(acc[0], acc[1]), a0, a1);
      l_run = l_run * alpha + (a0 + a1);
      // The output is divided by the sum of the weights that the product takes, the rounded ones, so that it is a
      // convex combination of the values (lse is of the unrounded sum). Added here, behind the hand-over, the
      // sum costs 5 % of a long call; in the loop above, 7 %.
      {
        float rnd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < kCols / 2; ++e) add_bf16x2_f32(rnd[2 * (e & 1)], rnd[2 * (e & 1) + 1], pk[e]);
        l_rnd = l_rnd * alpha + ((rnd[0] + rnd[1]) + (rnd[2] + rnd[3]));
      }
      m_run = m_new;
    }
    // The barrier of the rows' four warps has no limit of its own: whoever left early still comes to it for every
    // tile, or the others would wait there for ever. (They find out by their own waits. Agreeing at the barrier
    // to leave, by a reduction or a flag, takes 9 to 10 % of a long call.)
    for (; missed > 0; --missed) quarter_bar_sync(quarter);
    if (ok) ok = mbar_wait(&ctl.o_full, 0, wlim);
    const bool wok = __all_sync(0xffffffffu, ok);
    if (!wok && lane == 0) flag_timeout(p, ctl);
    ctl.red_sum[0][part4][t] = l_run;
    ctl.red_sum[1][part4][t] = l_rnd;
    all_bar_sync();
    auto row_sum = [&](int i) {
      return (ctl.red_sum[i][0][t] + ctl.red_sum[i][1][t]) + (ctl.red_sum[i][2][t] + ctl.red_sum[i][3][t]);
    };
    const float l = row_sum(0), l_out = row_sum(1);
    uint32_t rr[kOC];
    if (wok) {  // (whole warps: the loads from TMEM are theirs)
      tc_fence_after();
      tmem_load(tO + lane_off + part4 * kOC, rr);
      tmem_wait_ld();
      if (ctl.poison)
#pragma unroll
        for (int e = 0; e < kOC; ++e)
          rr[e] = __float_as_uint(poisoned(ctl, t, part4 * kOC + e, __uint_as_float(rr[e])));
    }
    if (p.nsplit > 1) {
      // this part of the keys: unnormalised output, reference maximum and sum
      float* slot = p.part + blockIdx.x * part_slot_floats(kBM, D);
      if (wok && seq >= 0) {
        uint4* o = reinterpret_cast<uint4*>(slot + t * D + part4 * kOC);
#pragma unroll
        for (int v = 0; v < kOC / 4; ++v) o[v] = make_uint4(rr[4 * v], rr[4 * v + 1], rr[4 * v + 2], rr[4 * v + 3]);
      }
      if (part4 == 0) {
        float* stat = slot + kBM * D;
        stat[t] = m_run == -INFINITY ? -INFINITY : m_run * sl;
        stat[kBM + t] = l;
        stat[4 * kBM + t] = l_out;
        reinterpret_cast<int64_t*>(stat + 2 * kBM)[t] = *abort_flag ? -1 : ctl.out_row[t];
      }
    } else {
      // O row / row sum -> bf16 into shared memory (the K stages are no longer read once o_full
      // has completed), 16-byte chunks XOR-swizzled by row; then the softmax threads store whole
      // rows, coalesced. Every softmax warp reaches the named barriers on every path.
      constexpr int kChunks = D / 8;  // 16-byte chunks per output row
      uint4* stage = reinterpret_cast<uint4*>(sK);  // 128 rows x D bf16 <= one K stage
      if (wok) {
        const float inv_l = 1.0f / l_out;
#pragma unroll
        for (int v = 0; v < kOC / 8; ++v) {
          uint4 u;
          u.x = pack_bf16x2(__uint_as_float(rr[8 * v + 0]) * inv_l, __uint_as_float(rr[8 * v + 1]) * inv_l);
          u.y = pack_bf16x2(__uint_as_float(rr[8 * v + 2]) * inv_l, __uint_as_float(rr[8 * v + 3]) * inv_l);
          u.z = pack_bf16x2(__uint_as_float(rr[8 * v + 4]) * inv_l, __uint_as_float(rr[8 * v + 5]) * inv_l);
          u.w = pack_bf16x2(__uint_as_float(rr[8 * v + 6]) * inv_l, __uint_as_float(rr[8 * v + 7]) * inv_l);
          const int chunk = part4 * (kChunks / kParts) + v;
          stage[t * kChunks + (chunk ^ (t & (kChunks - 1)))] = u;
        }
        if (p.lse && part4 == 0 && ctl.out_row[t] >= 0)
          p.lse[ctl.out_row[t]] = 0.69314718055994531f * (m_run * sl + log2f(l));
      }
      all_bar_sync();
      if (!*abort_flag) {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.a.o);
        const int tid = threadIdx.x;  // 0 .. 511
#pragma unroll 4
        for (int idx = tid; idx < kBM * kChunks; idx += 32 * kSoftmaxWarps) {
          const int row = idx / kChunks, chunk = idx % kChunks;
          if (ctl.out_row[row] >= 0)
            reinterpret_cast<uint4*>(out + ctl.out_row[row] * D)[chunk] =
                stage[row * kChunks + (chunk ^ (row & (kChunks - 1)))];
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kWPV) {
    if (lane == 0 && !mbar_wait(&ctl.drained, 0, wlim)) flag_timeout(p, ctl);
    __syncwarp();
    tc_fence_after();
    tmem_dealloc<kTmemCols>(ctl.tmem_base);
  }
}

// Joins the parts of a split launch: with M the largest reference maximum of a packed query,
// o = sum_c 2^(m_c - M) O_c / sum_c 2^(m_c - M) l'_c, l' the sum of the weights as O has them. kWarps warps
// share a query's parts, 32 at a time: a lane takes a part's factor and sums, then all take the parts' rows,
// coalesced. Bound by latency: one warp walking 33 parts of a row with a wait for each took 24 us, this 3
// beside the launch.
template <typename T, int D, int kWarps>
__global__ void __launch_bounds__(128, 6) prefix_join(const __grid_constant__ JoinParams p) {
  constexpr int kV = D / 32;  // elements per lane
  constexpr bool kRounded = sizeof(T) == 2;  // the output has its own sum
  __shared__ float s_o[4][D], s_top[4], s_l[4], s_lo[4];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % kWarps;
  const long long w = (static_cast<long long>(blockIdx.x) * 4 + warp) / kWarps;
  const bool in = w < p.rows;
  const int g = in ? static_cast<int>(w / p.queries) : 0, m = in ? static_cast<int>(w % p.queries) : 0;
  const int t = m % p.tile_rows;
  const size_t floats = part_slot_floats(p.tile_rows, D);
  const float* slot = p.part + (static_cast<size_t>(g) * p.tiles + m / p.tile_rows) * p.nsplit * floats;
  const float* stat = slot + p.tile_rows * D + t;
  grid_dep_wait();
  const int64_t row = reinterpret_cast<const int64_t*>(slot + (p.nsplit - 1) * floats +
                                                       p.tile_rows * (D + 2))[t];
  float top = -INFINITY, l = 0.f, lo = 0.f, o[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) o[e] = 0.f;
  const int c0 = p.nsplit * sub / kWarps, c1 = p.nsplit * (sub + 1) / kWarps;
  for (int c = c0; c < c1; c += 32) {
    const int n = min(32, c1 - c);
    const float mc = lane < n ? stat[(c + lane) * floats] : -INFINITY;
    const float lc = lane < n ? stat[(c + lane) * floats + p.tile_rows] : 0.f;
    const float lr = kRounded && lane < n ? stat[(c + lane) * floats + 4 * p.tile_rows] : 0.f;
    float most = fmaxf(top, mc);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
    // (A maximum of -inf: no key, or none with a weight, and a sum of 0; or, as maxima pass NaN over, scores
    // that are all NaN beside such keys, and a sum of NaN, which 0 times it lets through.)
    const float f = mc == -INFINITY ? 0.f : mc == most ? 1.f : ex2_approx(mc - most);
    const float back = top == -INFINITY ? 0.f : top == most ? 1.f : ex2_approx(top - most);
    float lf = f * lc, lof = f * lr;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) {
      lf += __shfl_xor_sync(0xffffffffu, lf, x);
      if (kRounded) lof += __shfl_xor_sync(0xffffffffu, lof, x);
    }
    l = l * back + lf;
    lo = lo * back + lof;
#pragma unroll
    for (int e = 0; e < kV; ++e) o[e] *= back;
    top = most;
#pragma unroll 8
    for (int u = 0; u < n; ++u) {
      const float fu = __shfl_sync(0xffffffffu, f, u);
      const float* src = slot + (c + u) * floats + t * D + lane * kV;
      if constexpr (kV == 4) {
        const float4 x = *reinterpret_cast<const float4*>(src);
        o[0] = fmaf(fu, x.x, o[0]);
        o[1] = fmaf(fu, x.y, o[1]);
        o[2] = fmaf(fu, x.z, o[2]);
        o[3] = fmaf(fu, x.w, o[3]);
      } else {
        const float2 x = *reinterpret_cast<const float2*>(src);
        o[0] = fmaf(fu, x.x, o[0]);
        o[1] = fmaf(fu, x.y, o[1]);
      }
    }
  }
  if (kWarps > 1) {
#pragma unroll
    for (int e = 0; e < kV; ++e) s_o[warp][lane * kV + e] = o[e];
    if (lane == 0) {
      s_top[warp] = top;
      s_l[warp] = l;
      s_lo[warp] = lo;
    }
    __syncthreads();
    if (sub != 0) return;
    float most = s_top[0];
#pragma unroll
    for (int k = 1; k < kWarps; ++k) most = fmaxf(most, s_top[k]);
    l = lo = 0.f;
#pragma unroll
    for (int e = 0; e < kV; ++e) o[e] = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float f = s_top[k] == -INFINITY ? 0.f : s_top[k] == most ? 1.f : ex2_approx(s_top[k] - most);
      l = fmaf(f, s_l[k], l);
      lo = fmaf(f, s_lo[k], lo);
#pragma unroll
      for (int e = 0; e < kV; ++e) o[e] = fmaf(f, s_o[k][lane * kV + e], o[e]);
    }
    top = most;
  }
  // (a row outside o: the workspace was changed under the call)
  if (!in || row < 0 || row >= p.out_rows) return;
  T* out = static_cast<T*>(p.o) + row * D + lane * kV;
  const float inv = 1.0f / (kRounded ? lo : l);
#pragma unroll
  for (int e = 0; e < kV; e += 2) {
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint32_t*>(out + e) = pack_bf16x2(o[e] * inv, o[e + 1] * inv);
    else
      *reinterpret_cast<float2*>(out + e) = make_float2(o[e] * inv, o[e + 1] * inv);
  }
  if (p.lse && lane == 0) p.lse[row] = 0.69314718055994531f * (top + log2f(l));
}

// ---------------------------------------------------------------- host side
constexpr int kSlots = 640;  // parts of a split launch at most

// CTAs per query tile. Costs in SM cycles: a CTA about `fixed` plus `step` per key tile; CTAs are alike,
// so that a launch takes as many rounds of them as the SMs need (measured: 112 tiles of 514 steps in 1,
// 2, 3, 4 and 5 parts take 399, 421, 428, 342 and 368 us); the join 5000 and 25 per part of a full
// tile.
int choose_split(long long items, int queries, double steps, int most, int sms) {
  constexpr double fixed = 12000, step = 1500;
  const double part = 25.0 * std::min(1.0, queries / static_cast<double>(kBM));
  int best = 1;
  double best_time = 0;
  for (int s = 1; s <= most && items * s <= kSlots; ++s) {
    const long long n = items * s;
    const double time = static_cast<double>((n + sms - 1) / sms) * (fixed + step * std::ceil(steps / s)) +
                        (s > 1 ? 5000.0 + part * static_cast<double>(n) : 0.0);
    if (s == 1 || time < best_time) {
      best = s;
      best_time = time;
    }
  }
  return best;
}

// The fp32 kernels: queries per CTA (8, two CTAs to an SM, or 128, one) and CTAs per query tile. Costs in
// SM cycles, fitted to 24 shapes (1 to 7168 packed queries, 3 to 1025 key tiles) with 1 to 152 parts, 8 % off
// on average: a CTA `fixed`, and per tile of 64 keys of 128 elements `tile`, a pair of the small ones
// together `pair`; the join 6000 and 9 per part. The choice is 0.3 % behind the best of all measured, 5 % at
// most. Measured with 4 kv heads, as 8 and as 128 queries: 7 queries over 4096 keys 10.8 and 37.7 us, 448 over
// 2048 83 and 86 us, 1792 over 2048 274 and 234 us.
int choose_f32(long long queries, int heads, int d, int steps, int sms, bool may_split, int& split) {
  int best = 0;
  double best_time = 0;
  for (const int rows : {kF32FewRows, kBM}) {
    const bool few = rows == kF32FewRows;
    const double width = d == 64 ? 0.64 : 1.0;
    const double tile = width * (few ? 3300 : 27000), pair = width * 5200, fixed = few ? 5500 : 25000;
    const long long items = (queries + rows - 1) / rows * heads;
    for (int s = 1;;) {
      const long long n = items * s, each = (n + sms - 1) / sms;
      const int part = (steps + s - 1) / s;
      const double single = fixed + part * tile;
      const double time = (few ? (each / 2) * (fixed + part * pair) + (each % 2) * single : each * single) +
                          (s > 1 ? 6000.0 + 9.0 * n : 0.0);
      if (best == 0 || time < best_time) {
        best = rows;
        split = s;
        best_time = time;
      }
      if (!may_split || part == 1) break;
      s = (steps + part - 2) / (part - 1);  // the fewest parts that are shorter
      if (items * s > kSlots) break;
    }
  }
  return best;
}

template <int D>
cudaError_t launch_tc(const PrefixParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap pk, pv, k, v;
  const AttnParams& a = p.a;
  if (!make_map3(&k, a.k, D, a.total_rows, a.hkv, static_cast<int64_t>(a.hkv) * D, D, kTN, 1) ||
      !make_map3(&v, a.v, D, a.total_rows, a.hkv, static_cast<int64_t>(a.hkv) * D, D, kTN, 1))
    return cudaErrorInvalidValue;
  if (p.prefix_len > 0) {
    if (!make_map3(&pk, p.pk, D, p.prefix_len, a.hkv, p.row_stride, p.head_stride, kTN, 1) ||
        !make_map3(&pv, p.pv, D, p.prefix_len, a.hkv, p.row_stride, p.head_stride, kTN, 1))
      return cudaErrorInvalidValue;
  } else {
    pk = k;
    pv = v;
  }
  cudaError_t e = ensure_smem_attr(prefix_tc<D>, smem_bytes<D>(), done);
  if (e != cudaSuccess) return e;
  const AttnLaunch L(static_cast<unsigned>(a.hkv * p.tiles * p.nsplit), kThreads, smem_bytes<D>(),
                     stream, 1, false);
  return cudaLaunchKernelEx(&L.cfg, prefix_tc<D>, p, pk, pv, k, v);
}

template <typename T, int D>
cudaError_t launch_join_d(const JoinParams& j, cudaStream_t stream) {
  if (j.nsplit > 8) {  // four warps to a query: its parts' rows are in flight together
    const AttnLaunch L(static_cast<unsigned>(j.rows), 128, 0, stream, 1, true);
    return cudaLaunchKernelEx(&L.cfg, prefix_join<T, D, 4>, j);
  }
  const AttnLaunch L(static_cast<unsigned>((j.rows + 3) / 4), 128, 0, stream, 1, true);
  return cudaLaunchKernelEx(&L.cfg, prefix_join<T, D, 1>, j);
}
template <typename T>
cudaError_t launch_join(const PrefixParams& p, int rows, cudaStream_t stream) {
  const JoinParams j{p.part, p.a.o, p.lse, static_cast<int64_t>(p.queries) * p.a.hkv,
                     static_cast<int64_t>(p.a.total_rows) * p.a.hq, p.queries, p.tiles, p.nsplit, rows};
  return p.a.head_dim == 64 ? launch_join_d<T, 64>(j, stream) : launch_join_d<T, 128>(j, stream);
}

dard_status prepare(const dard_prefix_attn_args* args, PrefixParams& p) {
  if (!args) return report(DARD_ERR_NULL, "args is NULL");
  const dard_attn_args& own = args->own;
  const dard_status st = prepare_attention(&own, p.a);
  if (st != DARD_OK) return st;
  if (own.rope_theta != 0.f)
    return report(DARD_ERR_VALUE, "rope_theta must be 0: q and k carry their positions");
  if (args->prefix_len < 0 || args->prefix_len > DARD_PREFIX_MAX_LEN)
    return report(DARD_ERR_SHAPE, "prefix_len %d outside 0..%d", args->prefix_len, DARD_PREFIX_MAX_LEN);
  const int esz = own.dtype == DARD_BF16 ? 2 : 4;
  if (args->prefix_len > 0) {
    if (!args->prefix_k || !args->prefix_v)
      return report(DARD_ERR_NULL, "prefix_k or prefix_v is NULL");
    if (args->prefix_row_stride < own.head_dim || args->prefix_head_stride < own.head_dim ||
        args->prefix_row_stride > (1ll << 36) || args->prefix_head_stride > (1ll << 36))
      return report(DARD_ERR_SHAPE, "prefix strides outside head_dim..2^36");
    if (((reinterpret_cast<uintptr_t>(args->prefix_k) | reinterpret_cast<uintptr_t>(args->prefix_v) |
          static_cast<uintptr_t>(args->prefix_row_stride * esz) |
          static_cast<uintptr_t>(args->prefix_head_stride * esz)) & 15u) != 0)
      return report(DARD_ERR_ALIGN, "prefix_k, prefix_v and their strides must be multiples of 16 bytes");
  }
  if ((reinterpret_cast<uintptr_t>(args->lse) & 3u) != 0)
    return report(DARD_ERR_ALIGN, "lse must be 4-byte aligned");
  p.pk = args->prefix_k;
  p.pv = args->prefix_v;
  p.row_stride = args->prefix_row_stride;
  p.head_stride = args->prefix_head_stride;
  p.prefix_len = args->prefix_len;
  p.lse = args->lse;
  p.group = own.hq / own.hkv;
  long long rows = 0;
  for (int s = 0; s < own.num_seqs; ++s) {
    p.q_before[s] = static_cast<int32_t>(rows);
    rows += p.a.seq[s].n_orig + p.a.seq[s].slen - p.a.seq[s].q_start;
  }
  p.q_before[own.num_seqs] = static_cast<int32_t>(rows);
  if (rows * p.group > (1ll << 31) - 256)
    return report(DARD_ERR_SHAPE, "query rows times heads of a group exceed 2^31 - 256");
  p.queries = static_cast<int32_t>(rows * p.group);
  const size_t need = dard_prefix_attention_workspace_size(p.a.total_rows, own.hq, own.hkv,
                                                           own.head_dim, args->prefix_len);
  if (args->workspace && args->workspace_bytes < need)
    return report(DARD_ERR_WORKSPACE, "workspace of %zu bytes needed", need);
  if ((reinterpret_cast<uintptr_t>(args->workspace) & 15u) != 0)
    return report(DARD_ERR_ALIGN, "workspace must be 16-byte aligned");
  p.part = static_cast<float*>(args->workspace);
  return DARD_OK;
}

}  // namespace
}  // namespace dard

extern "C" {

size_t dard_prefix_attention_workspace_size(int32_t total_rows, int32_t hq, int32_t hkv,
                                            int32_t head_dim, int32_t prefix_len) {
  using namespace dard;
  if (total_rows < 0 || hq < 1 || hkv < 1 || hq % hkv != 0 || (head_dim != 64 && head_dim != 128) ||
      prefix_len < 0 || prefix_len > DARD_PREFIX_MAX_LEN)
    return 0;
  return kSlots * part_slot_floats(kBM, head_dim) * sizeof(float);
}

dard_status dard_prefix_attention(const dard_prefix_attn_args* args, void* stream_ptr) {
  using namespace dard;
  report(DARD_OK, "%s", "");
  PrefixParams p;
  const dard_status st = prepare(args, p);
  if (st != DARD_OK) return st;
  if (p.queries == 0) return DARD_OK;
  const cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
  if (const char* w = std::getenv("DARD_TEST_WAIT_CYCLES")) p.a.wait_cycles = std::atoll(w);
  if (const char* d = std::getenv("DARD_TEST_DROP_KV")) p.a.test_drop_kv = std::atoi(d);
  if (std::getenv("DARD_TEST_FAIL_LAUNCH") != nullptr)
    return report(DARD_ERR_CUDA, "prefix attention launch failed: %s (DARD_TEST_FAIL_LAUNCH)",
                  cudaGetErrorString(cudaErrorLaunchFailure));
  const int sms = sm_count();
  const bool bf16 = args->own.dtype == DARD_BF16;
  const int key_tile = bf16 ? kTN : 64;
  // every tile has the prefix's key tiles and at least one of its own
  const int least = (p.prefix_len + key_tile - 1) / key_tile + 1;
  p.nsplit = 1;
  const int rows = bf16 ? kBM : choose_f32(p.queries, p.a.hkv, p.a.head_dim, least, sms,
                                           p.part != nullptr, p.nsplit);
  p.tiles = (p.queries + rows - 1) / rows;
  const long long items = static_cast<long long>(p.tiles) * p.a.hkv;
  if (items > (1ll << 31) - 1) return report(DARD_ERR_SHAPE, "too many query tiles");
  if (p.tiles <= kTileTable) {
    int s0 = 0, s1 = 0;
    double own = 0;  // own key tiles of a query tile, on average
    for (int i = 0; i < p.tiles; ++i) {
      const int t0 = static_cast<int>(static_cast<long long>(i) * rows / p.group);
      const int t1 = static_cast<int>((std::min<long long>((i + 1ll) * rows, p.queries) - 1) / p.group);
      while (p.q_before[s0 + 1] <= t0) ++s0;
      while (p.q_before[s1 + 1] <= t1) ++s1;
      p.tile_seq[i][0] = static_cast<uint8_t>(s0);
      p.tile_seq[i][1] = static_cast<uint8_t>(s1);
      own += (p.a.seq[s1].row_base + p.a.seq[s1].n_orig + p.a.seq[s1].slen - p.a.seq[s0].row_base +
              key_tile - 1) / key_tile;
    }
    if (bf16 && p.part != nullptr)
      p.nsplit = choose_split(items, p.queries, least - 1 + own / p.tiles, least, sms);
  }
  cudaError_t e;
  if (!bf16)
    e = launch_prefix_f32(p, rows, stream);
  else if (p.a.head_dim == 64)
    e = launch_tc<64>(p, stream);
  else
    e = launch_tc<128>(p, stream);
  if (e == cudaSuccess && p.nsplit > 1)
    e = bf16 ? launch_join<__nv_bfloat16>(p, rows, stream) : launch_join<float>(p, rows, stream);
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "prefix attention launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
