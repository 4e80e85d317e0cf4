// dard_prefix_f32.cu - attention over a shared prefix in fp32, on CUDA cores (dtype F32 of
// dard_prefix_attention). The same packed queries, key order and parts as the bf16 kernel
// (dard_prefix.cuh, dard_prefix_attn.cu), fp32 throughout.
//
// A CTA of 256 threads (16 x 16) holds 16 TR packed queries and takes 64 keys at a time through
// shared memory (cp.async, K of the next tile behind the products with V, V behind those with K).
// Thread (ty, tx) computes the scores of queries ty + 16 u and keys tx + 16 i, so that each 16-byte
// shared-memory load of a query or a key serves 4 or TR dot products; the 16 threads of a query
// share its maximum by shuffles, exchange the probabilities through shared memory within their
// half-warp, and add up columns 4 tx .. (and 64 + 4 tx ..) of its output.
// Bound by the fp32 FMA rate with TR = 8 (2048 rows x 28 heads over 4096 keys: 80 TFLOP/s); fewer queries
// take smaller tiles, which wait for shared memory (dard_prefix_attn.cu chooses).
#include <cfloat>

#include "dard_prefix.cuh"

namespace dard {
namespace {

constexpr int kF32Threads = 256;
constexpr int kF32Keys = 64;
constexpr int kPStride = kF32Keys + 16;  // the two half-warps' rows fall into different banks

template <int D, int TR>
constexpr size_t f32_smem() {
  return sizeof(float) * (16 * TR * D + 2 * kF32Keys * D + 16 * TR * kPStride) +
         sizeof(uint64_t) * 16 * TR;
}

template <int N>
__device__ __forceinline__ void cp_async_wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 16-byte chunk c of a row of D floats, in an order that puts neighbouring rows' equal chunks into
// different banks.
__device__ __forceinline__ int swz(int row, int c) { return c ^ (row & 7); }

template <int D, int TR>
__global__ void __launch_bounds__(kF32Threads) prefix_f32(const __grid_constant__ PrefixParams p) {
  constexpr int kRows = 16 * TR, kC = D / 4, kV = D / 64;
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

  // tile j of k (or v) into shared memory; rows behind the end are zeros
  auto load = [&](int j, bool is_k) {
    const bool own = j >= npt;
    const int row0 = own ? key0 + (j - npt) * kF32Keys : j * kF32Keys;
    const int end = own ? key_end : p.prefix_len;
    const float* src = static_cast<const float*>(own ? (is_k ? p.a.k : p.a.v) : (is_k ? p.pk : p.pv));
    const int64_t rs = own ? static_cast<int64_t>(p.a.hkv) * D : p.row_stride;
    const int64_t hs = own ? D : p.head_stride;
#pragma unroll
    for (int u = 0; u < kF32Keys * kC / kF32Threads; ++u) {
      const int i = tid + u * kF32Threads, r = i / kC, c = i % kC;
      const bool in = row0 + r < end;
      const float* from = src + (in ? (row0 + r) * rs + g * hs + 4 * c : 0);
      cp_async16((is_k ? sK + r * kC + swz(r, c) : sV + r * kC + c), from, in ? 16 : 0);
    }
    cp_async_commit();
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
  __shared__ BlockScratch scratch[(kRows + 31) / 32];
  if (tid < (kRows + 31) / 32 * 32 && j1 > npt) {
    const int warp_of_rows = tid / 32;
    int r = 0;
    if (tid < kRows && m0 + tid < p.queries) {
      const int tq = (m0 + tid) / p.group;
      seq = seq_of_query(p, tq, s0, s1 + 1);
      r = p.a.seq[seq].q_start + tq - p.q_before[seq];
    }
    __syncwarp();
    rm = warp_query_masks(p.a, scratch[warp_of_rows], seq, r, g == 0, store);
  }

  float m[TR], l[TR];
  float4 o[TR][kV];
#pragma unroll
  for (int u = 0; u < TR; ++u) {
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
    float s[TR][4];
#pragma unroll
    for (int u = 0; u < TR; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[u][i] = 0.f;
#pragma unroll 4
    for (int c = 0; c < kC; ++c) {
      float4 kf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) kf[i] = sK[(tx + 16 * i) * kC + swz(tx, c)];
#pragma unroll
      for (int u = 0; u < TR; ++u) {
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
    for (int u = 0; u < TR; ++u) {
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
        for (int u = 0; u < TR; ++u) {
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
      for (int u = 0; u < TR; ++u) {
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
  for (int u = 0; u < TR; ++u) {
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

template <int D, int TR>
cudaError_t launch(const PrefixParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = ensure_smem_attr(prefix_f32<D, TR>, f32_smem<D, TR>(), done);
  if (e != cudaSuccess) return e;
  const AttnLaunch L(static_cast<unsigned>(p.a.hkv * p.tiles * p.nsplit), kF32Threads,
                     f32_smem<D, TR>(), stream, 1, false);
  return cudaLaunchKernelEx(&L.cfg, prefix_f32<D, TR>, p);
}

template <int D>
cudaError_t launch_rows(const PrefixParams& p, int rows, cudaStream_t stream) {
  return rows == 16 ? launch<D, 1>(p, stream) : rows == 32 ? launch<D, 2>(p, stream) : launch<D, 8>(p, stream);
}

}  // namespace

cudaError_t launch_prefix_f32(const PrefixParams& p, int rows, cudaStream_t stream) {
  return p.a.head_dim == 64 ? launch_rows<64>(p, rows, stream) : launch_rows<128>(p, rows, stream);
}

}  // namespace dard
