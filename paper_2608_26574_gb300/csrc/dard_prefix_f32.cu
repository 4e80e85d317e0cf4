// dard_prefix_f32.cu - attention over a shared prefix in fp32, on CUDA cores (dtype F32 of
// dard_prefix_attention). The same packed queries, key order and parts as the bf16 kernel
// (dard_prefix.cuh, dard_prefix_attn.cu), fp32 throughout. Two kernels, for 128 packed queries to a CTA
// and for 8 (below); choose_f32 in dard_prefix_attn.cu takes the one that will be done first.
//
// Many queries: a CTA of 256 threads (16 x 16) holds 128 packed queries and takes 64 keys at a time
// through shared memory (cp.async, K of the next tile behind the products with V, V behind those with
// K). Thread (ty, tx) computes the scores of queries ty + 16 u and keys tx + 16 i, so that each 16-byte
// shared-memory load of a query or a key serves 4 or 8 dot products; the 16 threads of a query
// share its maximum by shuffles, exchange the probabilities through shared memory within their
// half-warp, and add up columns 4 tx .. (and 64 + 4 tx ..) of its output.
// In the products' loops the FMAs take twice the time of the shared-memory loads; around them eight warps hide
// neither the barriers nor the softmax. One sequence of 2048 rows, 28 heads on 4 of 128, over 4096 keys and its
// own rows: 4.26 ms, 180 GFLOP, 42 TFLOP/s, half of the FMA rate.
#include <cfloat>

#include "dard_prefix.cuh"

namespace dard {
namespace {

constexpr int kF32Threads = 256;
constexpr int kF32Keys = 64;
constexpr int kF32Rows = 128, kTR = kF32Rows / 16;  // a CTA's queries, and a thread's
constexpr int kPStride = kF32Keys + 16;  // the two half-warps' rows fall into different banks

template <int D>
constexpr size_t f32_smem() {
  return sizeof(float) * (kF32Rows * D + 2 * kF32Keys * D + kF32Rows * kPStride) +
         sizeof(uint64_t) * kF32Rows;
}

template <int N>
__device__ __forceinline__ void cp_async_wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 16-byte chunk c of a row of D floats, in an order that puts neighbouring rows' equal chunks into
// different banks.
__device__ __forceinline__ int swz(int row, int c) { return c ^ (row & 7); }

// Key tile j of k or v into shared memory, the chunks of a row in order or in swz() order; rows behind the
// end are zeros.
template <int D, bool kSwz>
__device__ __forceinline__ void load_tile(const PrefixParams& p, int g, int key0, int key_end, int npt, int j,
                                          bool is_k, float4* dst) {
  constexpr int kC = D / 4, kStep = kF32Threads / kC;  // rows between a thread's chunks
  static_assert(kStep % 8 == 0, "swz() is the same for all rows of a thread");
  const bool own = j >= npt;
  const int row0 = own ? key0 + (j - npt) * kF32Keys : j * kF32Keys;
  const int end = own ? key_end : p.prefix_len;
  const float* src = static_cast<const float*>(own ? (is_k ? p.a.k : p.a.v) : (is_k ? p.pk : p.pv));
  const int64_t rs = own ? static_cast<int64_t>(p.a.hkv) * D : p.row_stride;
  const int64_t hs = own ? D : p.head_stride;
  const int r = threadIdx.x / kC, c = threadIdx.x % kC;
  const float* from = src + (row0 + r) * rs + g * hs + 4 * c;
  dst += r * kC + (kSwz ? swz(r, c) : c);
  if (row0 + kF32Keys <= end) {
#pragma unroll
    for (int u = 0; u < kF32Keys / kStep; ++u)
      cp_async16(dst + u * kF32Threads, from + u * kStep * rs, 16);
  } else {
#pragma unroll
    for (int u = 0; u < kF32Keys / kStep; ++u) {
      const bool in = row0 + r + u * kStep < end;
      cp_async16(dst + u * kF32Threads, in ? from + u * kStep * rs : src, in ? 16 : 0);
    }
  }
  cp_async_commit();
}

template <int D>
__global__ void __launch_bounds__(kF32Threads) prefix_f32(const __grid_constant__ PrefixParams p) {
  constexpr int kRows = kF32Rows, kC = D / 4, kV = D / 64;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  float4* sQ = reinterpret_cast<float4*>(smem_raw);
  float4* sK = sQ + kRows * kC;
  float4* sV = sK + kF32Keys * kC;
  float* sP = reinterpret_cast<float*>(sV + kF32Keys * kC);
  uint64_t* sVis = reinterpret_cast<uint64_t*>(sP + kRows * kPStride);
  grid_dep_launch();
  const int item = blockIdx.x / p.nsplit, part = blockIdx.x % p.nsplit;
  const int g = item / p.tiles, m0 = item % p.tiles * kRows;
  int s0, s1, key0, key_end;
  own_range(p, item % p.tiles, kRows, s0, s1, key0, key_end);
  const int npt = (p.prefix_len + kF32Keys - 1) / kF32Keys;
  const int all = npt + (key_end - key0 + kF32Keys - 1) / kF32Keys;
  const int j0 = static_cast<int>(static_cast<long long>(all) * part / p.nsplit);
  const int j1 = static_cast<int>(static_cast<long long>(all) * (part + 1) / p.nsplit);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;

  auto load = [&](int j, bool is_k) {
    if (is_k)
      load_tile<D, true>(p, g, key0, key_end, npt, j, true, sK);
    else
      load_tile<D, false>(p, g, key0, key_end, npt, j, false, sV);
  };
  load(j0, true);
  load(j0, false);
  for (int i = tid; i < kRows * kC; i += kF32Threads) {
    const int t = i / kC, c = i % kC;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m0 + t < p.queries) {
      const int tq = (m0 + t) / p.group, s = seq_of_query(p, tq, s0, s1 + 1);
      const int64_t row = p.a.seq[s].row_base + p.a.seq[s].q_start + tq - p.q_before[s];
      v = __ldg(reinterpret_cast<const float4*>(p.a.q) +
                (row * p.a.hq + g * p.group + (m0 + t) % p.group) * kC + c);
    }
    sQ[t * kC + swz(t, c)] = v;
  }
  // thread t < kRows: query t's masks (while own tiles are to come)
  RowMasks rm{{0, 0}, {0, 0}};
  int seq = -1, store = 1;
  __shared__ BlockScratch scratch[kRows / 32];
  if (tid < kRows && j1 > npt) {
    const int warp_of_rows = tid / 32;
    int r = 0;
    if (m0 + tid < p.queries) {
      const int tq = (m0 + tid) / p.group;
      seq = seq_of_query(p, tq, s0, s1 + 1);
      r = p.a.seq[seq].q_start + tq - p.q_before[seq];
    }
    __syncwarp();
    rm = warp_query_masks(p.a, scratch[warp_of_rows], seq, r, g == 0, store);
  }

  float m[kTR], l[kTR];
  float4 o[kTR][kV];
#pragma unroll
  for (int u = 0; u < kTR; ++u) {
    m[u] = -INFINITY;
    l[u] = 0.f;
#pragma unroll
    for (int v = 0; v < kV; ++v) o[u][v] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const float sl = p.a.scale_log2;
  for (int j = j0; j < j1; ++j) {
    const bool own = j >= npt;
    if (tid < kRows)
      sVis[tid] = !own ? first64(p.prefix_len - j * kF32Keys)
                  : seq < 0 ? 0ull
                            : own_vis64(p.a.seq[seq], key0 + (j - npt) * kF32Keys - p.a.seq[seq].row_base, rm);
    cp_async_wait_group<1>();  // K_j
    __syncthreads();
    float s[kTR][4];
#pragma unroll
    for (int u = 0; u < kTR; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[u][i] = 0.f;
#pragma unroll 4
    for (int c = 0; c < kC; ++c) {
      float4 kf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) kf[i] = sK[(tx + 16 * i) * kC + swz(tx, c)];
#pragma unroll
      for (int u = 0; u < kTR; ++u) {
        const float4 qf = sQ[(ty + 16 * u) * kC + swz(ty, c)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[u][i] = fmaf(qf.x, kf[i].x, s[u][i]);
          s[u][i] = fmaf(qf.y, kf[i].y, s[u][i]);
          s[u][i] = fmaf(qf.z, kf[i].z, s[u][i]);
          s[u][i] = fmaf(qf.w, kf[i].w, s[u][i]);
        }
      }
    }
    __syncthreads();  // K_j has been read
    if (j + 1 < j1) load(j + 1, true); else cp_async_commit();
    // one step of the online softmax per query
#pragma unroll
    for (int u = 0; u < kTR; ++u) {
      const uint64_t vis = sVis[ty + 16 * u] >> tx;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[u][i] = (vis >> (16 * i)) & 1ull ? s[u][i] * sl : -INFINITY;
        top = fmaxf(top, s[u][i]);
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      if (top > m[u]) {
        const float alpha = exp2f(m[u] - top);  // 0 before the first key
        l[u] *= alpha;
#pragma unroll
        for (int v = 0; v < kV; ++v) {
          o[u][v].x *= alpha;
          o[u][v].y *= alpha;
          o[u][v].z *= alpha;
          o[u][v].w *= alpha;
        }
        m[u] = top;
      }
      const float ref = m[u] == -INFINITY ? 0.f : m[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = exp2f(s[u][i] - ref);
        l[u] += w;
        sP[(ty + 16 * u) * kPStride + tx + 16 * i] = w;
      }
    }
    cp_async_wait_group<1>();  // V_j
    bool bad = false;  // an own tile with values that are not finite
    if (own) {
#pragma unroll
      for (int u = 0; u < kF32Keys * kC / kF32Threads; ++u) {  // (what this thread copied)
        const float4 x = sV[tid + u * kF32Threads];
        bad |= !(fabsf(x.x) <= FLT_MAX && fabsf(x.y) <= FLT_MAX && fabsf(x.z) <= FLT_MAX && fabsf(x.w) <= FLT_MAX);
      }
    }
    if (own) bad = __syncthreads_or(bad); else __syncthreads();
    if (!bad) {
#pragma unroll 1
      for (int k = 0; k < kF32Keys; k += 4) {
        float4 vf[4][kV];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int v = 0; v < kV; ++v) vf[e][v] = sV[(k + e) * kC + tx + 16 * v];
#pragma unroll
        for (int u = 0; u < kTR; ++u) {
          const float4 w4 = *reinterpret_cast<const float4*>(sP + (ty + 16 * u) * kPStride + k);
          const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int v = 0; v < kV; ++v) {
              o[u][v].x = fmaf(w[e], vf[e][v].x, o[u][v].x);
              o[u][v].y = fmaf(w[e], vf[e][v].y, o[u][v].y);
              o[u][v].z = fmaf(w[e], vf[e][v].z, o[u][v].z);
              o[u][v].w = fmaf(w[e], vf[e][v].w, o[u][v].w);
            }
        }
      }
    } else {  // a key that a query does not see is left out (its weight is 0, its value may be NaN)
#pragma unroll
      for (int u = 0; u < kTR; ++u) {
        const uint64_t vis = sVis[ty + 16 * u];
#pragma unroll 4
        for (int k = 0; k < kF32Keys; ++k) {
          if (!((vis >> k) & 1ull)) continue;
          const float w = sP[(ty + 16 * u) * kPStride + k];
#pragma unroll
          for (int v = 0; v < kV; ++v) {
            const float4 x = sV[k * kC + tx + 16 * v];
            o[u][v].x = fmaf(w, x.x, o[u][v].x);
            o[u][v].y = fmaf(w, x.y, o[u][v].y);
            o[u][v].z = fmaf(w, x.z, o[u][v].z);
            o[u][v].w = fmaf(w, x.w, o[u][v].w);
          }
        }
      }
    }
    __syncthreads();  // V_j, the probabilities and sVis have been read
    if (j + 1 < j1) load(j + 1, false); else cp_async_commit();
  }
  // which queries are stored: in shared memory, over sVis
  if (tid < kRows) sVis[tid] = store;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kTR; ++u) {
    const int t = ty + 16 * u;
    float sum = l[u];
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    if (m0 + t >= p.queries) continue;
    const int tq = (m0 + t) / p.group, s = seq_of_query(p, tq, s0, s1 + 1);
    const int64_t row = sVis[t] == 0 ? -1
                            : (static_cast<int64_t>(p.a.seq[s].row_base) + p.a.seq[s].q_start + tq -
                               p.q_before[s]) * p.a.hq + g * p.group + (m0 + t) % p.group;
    if (p.nsplit > 1) {
      float* slot = p.part + blockIdx.x * part_slot_floats(kRows, D);
#pragma unroll
      for (int v = 0; v < kV; ++v)
        reinterpret_cast<float4*>(slot + t * D)[tx + 16 * v] = o[u][v];
      if (tx == 0) {
        float* stat = slot + kRows * D + t;
        stat[0] = m[u];
        stat[kRows] = sum;
        reinterpret_cast<int64_t*>(slot + kRows * (D + 2))[t] = row;
      }
    } else if (row >= 0) {
      float4* out = reinterpret_cast<float4*>(p.a.o) + row * kC;
      const float inv = 1.0f / sum;
#pragma unroll
      for (int v = 0; v < kV; ++v)
        out[tx + 16 * v] = make_float4(o[u][v].x * inv, o[u][v].y * inv, o[u][v].z * inv, o[u][v].w * inv);
      if (p.lse && tx == 0) p.lse[row] = 0.69314718055994531f * (m[u] + log2f(sum));
    }
  }
}

// ---------------------------------------------------------------- few queries
// Eight packed queries to a CTA: bytes, not products, are what they cost, and a shared-memory load takes
// its 512 bytes' time even where it is a broadcast. Scores: a half-warp takes a key, a thread every 16th
// chunk of it and of four queries, which stay in registers; 16 sums (four keys' with four queries) are
// added up over the half-warp by 15 shuffles that leave one to each thread (its registers hold them in an
// order of its own, the one that ends up in it first, so that no step has to select). Then warp r takes query
// r's online softmax step, its weights in place of the scores; products with V: thread (key group, column)
// adds eight queries' columns over its keys, and the groups are added up at the end.
// Two CTAs to an SM hide each other's waits; bound by the issue of instructions (a third of them FMAs) beside
// HBM: one token of 28 heads on 4 of 128 over 65536 keys (268 MB) 52 us, 40 at the copy's rate; with three
// CTAs of 80 registers 84, with bounds checked at every copy and selects in the shuffles' steps 73.
constexpr int kFewRows = kF32FewRows;
constexpr int kFewStride = kF32Keys + 4;  // of a row of scores

template <int D>
constexpr size_t few_smem() {
  return sizeof(float) * (2 * kF32Keys * D + kFewRows * D + kFewRows * kFewStride + 2 * kFewRows) +
         sizeof(uint64_t) * kFewRows;
}

__device__ __forceinline__ void add_scaled(float4& o, float w, const float4& v) {
  o.x = fmaf(w, v.x, o.x);
  o.y = fmaf(w, v.y, o.y);
  o.z = fmaf(w, v.z, o.z);
  o.w = fmaf(w, v.w, o.w);
}

template <int D>
__global__ void __launch_bounds__(kF32Threads, 2) prefix_f32_few(const __grid_constant__ PrefixParams p) {
  constexpr int kC = D / 4, kGroups = kF32Threads / kC, kGroupKeys = kF32Keys / kGroups;
  static_assert(kF32Threads == 4 * kF32Keys && kFewRows * 32 == kF32Threads && kGroupKeys % 4 == 0,
                "the threads' roles");
  extern __shared__ __align__(16) uint8_t smem_raw[];
  float4* sK = reinterpret_cast<float4*>(smem_raw);
  float4* sV = sK + kF32Keys * kC;
  float4* sQ = sV + kF32Keys * kC;
  float* sS = reinterpret_cast<float*>(sQ + kFewRows * kC);  // [row][key]: scores, then weights
  float* sAlpha = sS + kFewRows * kFewStride;
  float* sL = sAlpha + kFewRows;
  uint64_t* sVis = reinterpret_cast<uint64_t*>(sL + kFewRows);
  __shared__ BlockScratch scratch;
  grid_dep_launch();
  const int item = blockIdx.x / p.nsplit, part = blockIdx.x % p.nsplit;
  const int g = item / p.tiles, m0 = item % p.tiles * kFewRows;
  int s0, s1, key0, key_end;
  own_range(p, item % p.tiles, kFewRows, s0, s1, key0, key_end);
  const int npt = (p.prefix_len + kF32Keys - 1) / kF32Keys;
  const int all = npt + (key_end - key0 + kF32Keys - 1) / kF32Keys;
  const int j0 = static_cast<int>(static_cast<long long>(all) * part / p.nsplit);
  const int j1 = static_cast<int>(static_cast<long long>(all) * (part + 1) / p.nsplit);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  load_tile<D, false>(p, g, key0, key_end, npt, j0, true, sK);
  load_tile<D, false>(p, g, key0, key_end, npt, j0, false, sV);
  for (int i = tid; i < kFewRows * kC; i += kF32Threads) {
    const int t = i / kC;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m0 + t < p.queries) {
      const int tq = (m0 + t) / p.group, s = seq_of_query(p, tq, s0, s1 + 1);
      const int64_t row = p.a.seq[s].row_base + p.a.seq[s].q_start + tq - p.q_before[s];
      v = __ldg(reinterpret_cast<const float4*>(p.a.q) +
                (row * p.a.hq + g * p.group + (m0 + t) % p.group) * kC + i % kC);
    }
    sQ[i] = v;
  }
  // thread t < kFewRows: query t's masks (while own tiles are to come)
  RowMasks rm{{0, 0}, {0, 0}};
  int seq = -1, store = 1;
  if (warp == 0 && j1 > npt) {
    int r = 0;
    if (tid < kFewRows && m0 + tid < p.queries) {
      const int tq = (m0 + tid) / p.group;
      seq = seq_of_query(p, tq, s0, s1 + 1);
      r = p.a.seq[seq].q_start + tq - p.q_before[seq];
    }
    __syncwarp();
    rm = warp_query_masks(p.a, scratch, seq, r, g == 0, store);
  }

  // scores: queries row0 .. row0 + 3, keys lane_key .. lane_key + 7
  const int slice = lane % 16, row0 = warp / 4 * 4, lane_key = warp % 4 * 16 + lane / 16 * 8;
  const int col = tid % kC, grp = tid / kC;
  float m = -INFINITY, l = 0.f;  // of query `warp`: the same in every lane; this lane's share
  float4 o[kFewRows];            // of column `col`, over the keys of group `grp`
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();  // the queries are there
  float4 q[4][kC / 16];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < kC / 16; ++i) q[r][i] = sQ[(row0 + (r ^ (slice / 4))) * kC + slice + 16 * i];
  const float sl = p.a.scale_log2;
  for (int j = j0; j < j1; ++j) {
    const bool own = j >= npt;
    if (tid < kFewRows)
      sVis[tid] = !own ? first64(p.prefix_len - j * kF32Keys)
                  : seq < 0 ? 0ull
                            : own_vis64(p.a.seq[seq], key0 + (j - npt) * kF32Keys - p.a.seq[seq].row_base, rm);
    cp_async_wait_group<1>();  // K_j
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 8; b += 4) {
      float s[16];  // [query ^ (slice / 4)][key ^ (slice % 4)]
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[4 * r + k] = 0.f;
#pragma unroll
        for (int i = 0; i < kC / 16; ++i) {
          const float4 kf = sK[(lane_key + b + (k ^ (slice % 4))) * kC + slice + 16 * i];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[4 * r + k] = fmaf(q[r][i].x, kf.x, s[4 * r + k]);
            s[4 * r + k] = fmaf(q[r][i].y, kf.y, s[4 * r + k]);
            s[4 * r + k] = fmaf(q[r][i].z, kf.z, s[4 * r + k]);
            s[4 * r + k] = fmaf(q[r][i].w, kf.w, s[4 * r + k]);
          }
        }
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1)
#pragma unroll
        for (int i = 0; i < x; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i + x], x);
      sS[(row0 + slice / 4) * kFewStride + lane_key + b + slice % 4] = s[0];
    }
    __syncthreads();  // the scores are there, K_j has been read
    if (j + 1 < j1) load_tile<D, false>(p, g, key0, key_end, npt, j + 1, true, sK); else cp_async_commit();
    {
      const uint64_t vis = sVis[warp];
      float* const row = sS + warp * kFewStride + lane;
      float z[2], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        z[i] = (vis >> (lane + 32 * i)) & 1ull ? row[32 * i] * sl : -INFINITY;
        top = fmaxf(top, z[i]);
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float alpha = top > m ? exp2f(m - top) : 1.f;  // 0 before the first key
      if (top > m) m = top;
      const float ref = m == -INFINITY ? 0.f : m;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float w = exp2f(z[i] - ref);
        l += w;
        row[32 * i] = w;
      }
      if (lane == 0) sAlpha[warp] = alpha;
    }
    cp_async_wait_group<1>();  // V_j
    bool bad = false;  // an own tile with values that are not finite
    if (own) {
#pragma unroll
      for (int u = 0; u < kF32Keys * kC / kF32Threads; ++u) {  // (what this thread copied)
        const float4 x = sV[tid + u * kF32Threads];
        bad |= !(fabsf(x.x) <= FLT_MAX && fabsf(x.y) <= FLT_MAX && fabsf(x.z) <= FLT_MAX && fabsf(x.w) <= FLT_MAX);
      }
    }
    if (own) bad = __syncthreads_or(bad); else __syncthreads();
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
      const float alpha = sAlpha[r];
      o[r].x *= alpha;
      o[r].y *= alpha;
      o[r].z *= alpha;
      o[r].w *= alpha;
    }
    if (!bad) {
#pragma unroll
      for (int k = grp * kGroupKeys; k < (grp + 1) * kGroupKeys; k += 4) {
        float4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = sV[(k + i) * kC + col];
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
          const float4 w4 = *reinterpret_cast<const float4*>(sS + r * kFewStride + k);
          add_scaled(o[r], w4.x, v[0]);
          add_scaled(o[r], w4.y, v[1]);
          add_scaled(o[r], w4.z, v[2]);
          add_scaled(o[r], w4.w, v[3]);
        }
      }
    } else {  // a hidden key is left out, as its value may be NaN: its weight is 0
#pragma unroll 1
      for (int k = grp * kGroupKeys; k < (grp + 1) * kGroupKeys; ++k) {
        const float4 v = sV[k * kC + col];
#pragma unroll
        for (int r = 0; r < kFewRows; ++r)
          if ((sVis[r] >> k) & 1ull) add_scaled(o[r], sS[r * kFewStride + k], v);
      }
    }
    __syncthreads();  // V_j, the weights and sVis have been read
    if (j + 1 < j1) load_tile<D, false>(p, g, key0, key_end, npt, j + 1, false, sV); else cp_async_commit();
  }
  cp_async_wait_group<0>();
  // which queries are stored, the sums, and the groups' outputs, added up in order
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
  if (lane == 0) {
    sL[warp] = l;
    sAlpha[warp] = m;
  }
  if (tid < kFewRows) sVis[tid] = store;
  float4* sO = sK;  // [group][row][column], over K and V
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) sO[(grp * kFewRows + r) * kC + col] = o[r];
  __syncthreads();
  for (int i = tid; i < kFewRows * kC; i += kF32Threads) {
    const int t = i / kC, c = i % kC;
    if (m0 + t >= p.queries) continue;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const float4 x = sO[(k * kFewRows + t) * kC + c];
      sum.x += x.x;
      sum.y += x.y;
      sum.z += x.z;
      sum.w += x.w;
    }
    const int tq = (m0 + t) / p.group, s = seq_of_query(p, tq, s0, s1 + 1);
    const int64_t row = sVis[t] == 0 ? -1
                            : (static_cast<int64_t>(p.a.seq[s].row_base) + p.a.seq[s].q_start + tq -
                               p.q_before[s]) * p.a.hq + g * p.group + (m0 + t) % p.group;
    if (p.nsplit > 1) {
      float* slot = p.part + blockIdx.x * part_slot_floats(kFewRows, D);
      reinterpret_cast<float4*>(slot + t * D)[c] = sum;
      if (c == 0) {
        float* stat = slot + kFewRows * D + t;
        stat[0] = sAlpha[t];
        stat[kFewRows] = sL[t];
        reinterpret_cast<int64_t*>(slot + kFewRows * (D + 2))[t] = row;
      }
    } else if (row >= 0) {
      const float inv = 1.0f / sL[t];
      (reinterpret_cast<float4*>(p.a.o) + row * kC)[c] =
          make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
      if (p.lse && c == 0) p.lse[row] = 0.69314718055994531f * (sAlpha[t] + log2f(sL[t]));
    }
  }
}

template <int D>
cudaError_t launch_many(const PrefixParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = ensure_smem_attr(prefix_f32<D>, f32_smem<D>(), done);
  if (e != cudaSuccess) return e;
  const AttnLaunch L(static_cast<unsigned>(p.a.hkv * p.tiles * p.nsplit), kF32Threads, f32_smem<D>(), stream, 1,
                     false);
  return cudaLaunchKernelEx(&L.cfg, prefix_f32<D>, p);
}

template <int D>
cudaError_t launch_few(const PrefixParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = ensure_smem_attr(prefix_f32_few<D>, few_smem<D>(), done);
  if (e != cudaSuccess) return e;
  const AttnLaunch L(static_cast<unsigned>(p.a.hkv * p.tiles * p.nsplit), kF32Threads, few_smem<D>(), stream, 1,
                     false);
  return cudaLaunchKernelEx(&L.cfg, prefix_f32_few<D>, p);
}

template <int D>
cudaError_t launch_rows(const PrefixParams& p, int rows, cudaStream_t stream) {
  return rows == kFewRows ? launch_few<D>(p, stream) : launch_many<D>(p, stream);
}

}  // namespace

cudaError_t launch_prefix_f32(const PrefixParams& p, int rows, cudaStream_t stream) {
  return p.a.head_dim == 64 ? launch_rows<64>(p, rows, stream) : launch_rows<128>(p, rows, stream);
}

}  // namespace dard
