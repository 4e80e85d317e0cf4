// dard_norm.cu - dard_residual_norm (residual addition, root-mean-square norm, optional MXFP8
// output) and dard_mx_quantize (the MXFP8 rounding alone).
//
// Both are bound by HBM: every input byte is read once, every output byte written once, and
// a row stays in registers between the sum of its squares and its scaling. On GB300 38912 rows of
// 4096 bf16 with every output (1.44 GB) take 207 us, 6.95 TB/s, and the MXFP8 rounding of
// 64 x 2048 x 2048 bf16 (0.81 GB) 127 us, 6.4 TB/s; a plain copy moves 6.8. One row of 4096 takes
// 2.8 us, its chain of latencies (loads, two reductions, stores).
#include <cuda_bf16.h>

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

// ---------------------------------------------------------------- element access
// Eight consecutive elements as fp32, from / to 16-byte aligned memory. (Plain loads: an
// output may be written over its input.)
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    const float4 a = reinterpret_cast<const float4*>(p)[0];
    const float4 b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]),
                                              bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
// Rounding to T and back: the value a later read of the stored element gives.
template <typename T>
__device__ __forceinline__ float rounded(float v) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(__float2bfloat16_rn(v));
  return v;
}
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float v) { d = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f(float& d, float v) { d = v; }

struct NormParams {
  const void* x;
  const void* delta;
  const void* weight;
  void* residual;
  void* y;
  uint8_t* y8;
  uint8_t* y8_scale;
  int64_t rows, x_stride, delta_stride, residual_stride, y_stride, y8_stride, scale_stride;
  int32_t dim;
  float eps, inv_dim;
};

// The sum of `v` over a row's threads: `kWarps` warps of the CTA (1: a row per warp).
template <int kWarps>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (kWarps == 1) return v;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = (threadIdx.x & 31) < kWarps ? red[threadIdx.x & 31] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One row per kWarps warps; a thread holds kVec runs of eight consecutive elements, run j of
// thread t at element 8 (t + j threads). Four neighbouring threads hold one MX block. The sum of
// squares is fp32, eight to 32 elements in a thread's chain, then a tree.
template <typename T, int kWarps, int kVec>
__global__ void __launch_bounds__(kWarps == 1 ? 128 : 32 * kWarps)
    norm_rows(const __grid_constant__ NormParams p) {
  constexpr int kThreads = 32 * kWarps;
  constexpr int kRows = kWarps == 1 ? 4 : 1;  // rows per CTA
  __shared__ float red[32];
  const int t = kWarps == 1 ? threadIdx.x & 31 : threadIdx.x;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows +
                      (kWarps == 1 ? threadIdx.x >> 5 : 0);
  if (row >= p.rows) return;  // kRows > 1: a whole warp leaves
  const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
  const T* delta = p.delta ? static_cast<const T*>(p.delta) + row * p.delta_stride : nullptr;
  float v[kVec][8];
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const int e = 8 * (t + j * kThreads);
    if (e < p.dim) {
      load8(x + e, v[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
    }
  }
  if (delta != nullptr) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int e = 8 * (t + j * kThreads);
      if (e < p.dim) {
        float d[8];
        load8(delta + e, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = rounded<T>(v[j][i] + d[i]);
      }
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(v[j][i], v[j][i], sum);
  }
  if (p.residual != nullptr) {
    T* r = static_cast<T*>(p.residual) + row * p.residual_stride;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int e = 8 * (t + j * kThreads);
      if (e < p.dim) store8(r + e, v[j]);
    }
  }
  sum = row_sum<kWarps>(sum, red);
  const float inv = rsqrtf(sum * p.inv_dim + p.eps);
  T* y = p.y ? static_cast<T*>(p.y) + row * p.y_stride : nullptr;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const int e = 8 * (t + j * kThreads);
    const bool in = e < p.dim;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] *= inv;
    if (p.weight != nullptr && in) {
      float w[8];
      load8(static_cast<const T*>(p.weight) + e, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= w[i];
    }
    if (y != nullptr && in) store8(y + e, v[j]);
    if (p.y8 != nullptr) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max_nan(m, fabsf(v[j][i]));
      m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const uint32_t b = mx_scale_byte(m);
      const float s = mx_inverse(b);
      if (in) {
        uint2 c;
        c.x = e4m3x4(v[j][0] * s, v[j][1] * s, v[j][2] * s, v[j][3] * s);
        c.y = e4m3x4(v[j][4] * s, v[j][5] * s, v[j][6] * s, v[j][7] * s);
        *reinterpret_cast<uint2*>(p.y8 + row * p.y8_stride + e) = c;
        if ((t & 3) == 0)
          p.y8_scale[row * p.scale_stride + e / kMxBlock] = static_cast<uint8_t>(b);
      }
    }
  }
}

// The same for rows that 16-byte accesses cannot take (an odd dim, stride or address): one
// row per CTA of kWarps warps, element t + j threads of the row with thread t, so that a warp
// accesses 32 consecutive elements and holds one MX block. 1777 x 2731 fp32 (78 MB)
// takes 15 us. Where norm_rows can be used it is the faster one: 38912 x 4096 bf16 207 us
// against 438 here, whose accesses are an eighth as wide, so that it is bound by their number.
template <typename T, int kWarps, int kElems>
__global__ void __launch_bounds__(32 * kWarps) norm_rows_any(const __grid_constant__ NormParams p) {
  constexpr int kThreads = 32 * kWarps;
  __shared__ float red[32];
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
  float v[kElems];
#pragma unroll
  for (int j = 0; j < kElems; ++j) {
    const int e = t + j * kThreads;
    v[j] = e < p.dim ? to_f(x[e]) : 0.f;
  }
  if (p.delta != nullptr) {
    const T* delta = static_cast<const T*>(p.delta) + row * p.delta_stride;
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      const int e = t + j * kThreads;
      if (e < p.dim) v[j] = rounded<T>(v[j] + to_f(delta[e]));
    }
  }
  const T* weight = static_cast<const T*>(p.weight);
  constexpr bool kEarly = kElems <= 16;  // (more do not fit the registers)
  T w[kElems];  // on its way during the reduction
  if (kEarly && weight != nullptr) {
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      const int e = t + j * kThreads;
      if (e < p.dim) w[j] = weight[e];
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < kElems; ++j) sum = fmaf(v[j], v[j], sum);
  if (p.residual != nullptr) {
    T* r = static_cast<T*>(p.residual) + row * p.residual_stride;
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      const int e = t + j * kThreads;
      if (e < p.dim) from_f(r[e], v[j]);
    }
  }
  sum = row_sum<kWarps>(sum, red);
  const float inv = rsqrtf(sum * p.inv_dim + p.eps);
  T* y = p.y ? static_cast<T*>(p.y) + row * p.y_stride : nullptr;
#pragma unroll
  for (int j = 0; j < kElems; ++j) {
    const int e = t + j * kThreads;
    const bool in = e < p.dim;
    v[j] *= inv;
    if (weight != nullptr && in) v[j] *= to_f(kEarly ? w[j] : weight[e]);
    if (y != nullptr && in) from_f(y[e], v[j]);
    if (p.y8 != nullptr) {
      float m = fabsf(v[j]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
      const uint32_t b = mx_scale_byte(m);
      if (in) {
        p.y8[row * p.y8_stride + e] = static_cast<uint8_t>(e4m3x2(v[j] * mx_inverse(b), 0.f));
        if ((t & 31) == 0)
          p.y8_scale[row * p.scale_stride + e / kMxBlock] = static_cast<uint8_t>(b);
      }
    }
  }
}

template <typename T>
cudaError_t launch_norm(const NormParams& p, bool vec, cudaStream_t s) {
  const unsigned rows = static_cast<unsigned>(p.rows);
  const int d = p.dim;
  if (vec) {
    // A row per warp up to 1024 elements; then as few warps as hold the row in two runs of
    // eight per thread, four runs for the longest rows: enough loads in flight with few threads
    // in a row's two barriers. bf16 with MXFP8, us, against other splits (warps x runs): 512: 46,
    // 4 x 1 71; 1024: 97, 4 x 1 96; 2048: 174, 1 x 8 243, 8 x 1 193; 4096: 207, 4 x 4 222, 16 x 1
    // 240; 8192: 182, 8 x 4 195, 32 x 1 217; 16384: 218, 32 x 2 258.
    if (d <= 512) norm_rows<T, 1, 2><<<(rows + 3) / 4, 128, 0, s>>>(p);
    else if (d <= 1024) norm_rows<T, 1, 4><<<(rows + 3) / 4, 128, 0, s>>>(p);
    else if (d <= 2048) norm_rows<T, 4, 2><<<rows, 128, 0, s>>>(p);
    else if (d <= 4096) norm_rows<T, 8, 2><<<rows, 256, 0, s>>>(p);
    else if (d <= 8192) norm_rows<T, 16, 2><<<rows, 512, 0, s>>>(p);
    else if (d <= 16384) norm_rows<T, 16, 4><<<rows, 512, 0, s>>>(p);
    else norm_rows<T, 32, 4><<<rows, 1024, 0, s>>>(p);
  } else {
    // The fewest warps that hold the row in eight elements per thread (1777 x 2731 fp32: 12
    // warps 14.9 us, 8 of sixteen elements 15.6, 16 15.5, 32 of four 17.7).
    if (d <= 4 * 32 * 8) norm_rows_any<T, 4, 8><<<rows, 4 * 32, 0, s>>>(p);
    else if (d <= 8 * 32 * 8) norm_rows_any<T, 8, 8><<<rows, 8 * 32, 0, s>>>(p);
    else if (d <= 12 * 32 * 8) norm_rows_any<T, 12, 8><<<rows, 12 * 32, 0, s>>>(p);
    else if (d <= 16 * 32 * 8) norm_rows_any<T, 16, 8><<<rows, 16 * 32, 0, s>>>(p);
    else if (d <= 32 * 32 * 8) norm_rows_any<T, 32, 8><<<rows, 32 * 32, 0, s>>>(p);
    else if (d <= 32 * 32 * 16) norm_rows_any<T, 32, 16><<<rows, 32 * 32, 0, s>>>(p);
    else norm_rows_any<T, 32, 32><<<rows, 32 * 32, 0, s>>>(p);
  }
  return cudaGetLastError();
}

// ---------------------------------------------------------------- MXFP8 rounding
struct MxParams {
  const void* x;
  uint8_t* codes;
  uint8_t* scales;
  int64_t rows, total_rows;           // rows of a matrix, of all matrices
  int64_t x_row_stride, x_batch_stride, scale_stride;
  int64_t tiles_per_matrix;           // layout TILES
  int32_t cols, tile_cols, layout;
  int32_t runs;                       // cols / 16
  int32_t one;                        // a single matrix (or a batch that is laid out as one)
};

__device__ __forceinline__ uint8_t* scale_at(const MxParams& p, int64_t row, int block) {
  if (p.layout == DARD_MX_SCALE_ROWS) return p.scales + row * p.scale_stride + block;
  const int64_t b = p.one ? 0 : row / p.rows, r = row - b * p.rows;
  return p.scales + (b * p.tiles_per_matrix + r / 128 * p.tile_cols + block / 4) * kMxTileBytes +
         mx_tile_byte(static_cast<int>(r % 128), block);
}
template <typename T>
__device__ __forceinline__ const T* row_at(const MxParams& p, int64_t row) {
  const int64_t b = p.one ? 0 : row / p.rows;
  return static_cast<const T*>(p.x) + b * p.x_batch_stride + (row - b * p.rows) * p.x_row_stride;
}

// Sixteen consecutive elements from 16-byte aligned memory, as they are; their largest magnitude
// (bf16: pair by pair); element i as fp32.
template <typename T>
__device__ __forceinline__ void load16(const T* p, uint32_t (&raw)[sizeof(T) * 4]) {
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) {
    const uint4 u = reinterpret_cast<const uint4*>(p)[i];
    raw[4 * i] = u.x;
    raw[4 * i + 1] = u.y;
    raw[4 * i + 2] = u.z;
    raw[4 * i + 3] = u.w;
  }
}
template <typename T>
__device__ __forceinline__ float largest16(const uint32_t (&raw)[sizeof(T) * 4]) {
  if constexpr (sizeof(T) == 2) {
    uint32_t m = raw[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 8; ++i)
      asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(raw[i] & 0x7fff7fffu));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    float m = fabsf(__uint_as_float(raw[0]));
#pragma unroll
    for (int i = 1; i < 16; ++i) m = max_nan(m, fabsf(__uint_as_float(raw[i])));
    return m;
  }
}
template <typename T>
__device__ __forceinline__ float element16(const uint32_t (&raw)[sizeof(T) * 4], int i) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
  else
    return __uint_as_float(raw[i]);
}

// Runs of 16 elements: run i of the batch is run i % runs of row i / runs. A thread takes runs
// 256 apart, kSteps of them in flight; two neighbouring threads hold one block. What costs here
// is instructions: eight elements per run and a division for each took 272 us at 64 x 2048 x 2048
// bf16, where the bytes take 120 and this takes 127.
template <typename T, int kSteps>
__global__ void __launch_bounds__(256) mx_rows(const __grid_constant__ MxParams p) {
  const int64_t first = static_cast<int64_t>(blockIdx.x) * 256 * kSteps + threadIdx.x;
  const int row_step = 256 / p.runs, run_step = 256 % p.runs;
  uint32_t raw[kSteps][sizeof(T) * 4];
  int64_t row[kSteps];
  int run[kSteps];
  row[0] = first < 0xffffffffll ? static_cast<uint32_t>(first) / static_cast<uint32_t>(p.runs)
                                : first / p.runs;
  run[0] = static_cast<int>(first - row[0] * p.runs);
#pragma unroll
  for (int j = 1; j < kSteps; ++j) {
    row[j] = row[j - 1] + row_step;
    run[j] = run[j - 1] + run_step;
    if (run[j] >= p.runs) {
      run[j] -= p.runs;
      ++row[j];
    }
  }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    if (row[j] < p.total_rows) {
      load16<T>(row_at<T>(p, row[j]) + 16 * run[j], raw[j]);
    } else {
#pragma unroll
      for (int k = 0; k < static_cast<int>(sizeof(T)) * 4; ++k) raw[j][k] = 0;
    }
  }
  // whole tiles of four blocks: eight threads hold one, whose four bytes lie side by side
  const bool by_four = p.cols % 128 == 0;
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    float m = largest16<T>(raw[j]);
    m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const uint32_t b = mx_scale_byte(m);
    const float s = mx_inverse(b);
    uint32_t four = b | __shfl_down_sync(0xffffffffu, b, 2) << 8;
    four |= __shfl_down_sync(0xffffffffu, four, 4) << 16;
    if (row[j] < p.total_rows) {
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        c[i] = e4m3x4(element16<T>(raw[j], 4 * i) * s, element16<T>(raw[j], 4 * i + 1) * s,
                      element16<T>(raw[j], 4 * i + 2) * s, element16<T>(raw[j], 4 * i + 3) * s);
      *reinterpret_cast<uint4*>(p.codes + row[j] * p.cols + 16 * run[j]) =
          make_uint4(c[0], c[1], c[2], c[3]);
      if (by_four) {
        if ((threadIdx.x & 7) == 0)
          *reinterpret_cast<uint32_t*>(scale_at(p, row[j], run[j] / 2)) = four;
      } else if ((threadIdx.x & 1) == 0) {
        *scale_at(p, row[j], run[j] / 2) = static_cast<uint8_t>(b);
      }
    }
  }
}

// Rows that 16-byte accesses cannot take: one block per warp, one element per lane, bound by the
// instructions around each block (64 x 2048 x 2048 bf16 would take 1.2 ms this way).
template <typename T>
__global__ void __launch_bounds__(256) mx_rows_any(const __grid_constant__ MxParams p) {
  const int lane = threadIdx.x & 31, blocks = p.cols / kMxBlock;
  const int64_t total = p.total_rows * blocks;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5); i < total;
       i += static_cast<int64_t>(gridDim.x) * 8) {
    const int64_t row = i / blocks;
    const int block = static_cast<int>(i % blocks);
    const float v = to_f(row_at<T>(p, row)[block * kMxBlock + lane]);
    float m = fabsf(v);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    const uint32_t b = mx_scale_byte(m);
    p.codes[row * p.cols + block * kMxBlock + lane] =
        static_cast<uint8_t>(e4m3x2(v * mx_inverse(b), 0.f));
    if (lane == 0) *scale_at(p, row, block) = static_cast<uint8_t>(b);
  }
}

template <typename T>
cudaError_t launch_mx(const MxParams& p, bool vec, cudaStream_t s) {
  if (vec) {
    // Four runs of bf16 in flight: 128 us at 64 x 2048 x 2048 (two 136, eight 155: registers);
    // two of fp32, as many bytes: 96 us at 32 x 2048 x 2048 (one 94, four 111).
    constexpr int kSteps = sizeof(T) == 2 ? 4 : 2;
    const int64_t runs = p.total_rows * p.runs;
    const int64_t ctas = (runs + 256 * kSteps - 1) / (256 * kSteps);
    if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
    mx_rows<T, kSteps><<<static_cast<unsigned>(ctas), 256, 0, s>>>(p);
  } else {
    const int64_t warps = p.total_rows * (p.cols / kMxBlock);
    const int64_t ctas = std::min<int64_t>((warps + 7) / 8, 16ll * sm_count());
    mx_rows_any<T><<<static_cast<unsigned>(ctas), 256, 0, s>>>(p);
  }
  return cudaGetLastError();
}

bool multiple(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Test hook (failure-path tests; unset in normal operation): a launch that reports failure
// without launching.
bool fail_launch() { return std::getenv("DARD_TEST_FAIL_LAUNCH") != nullptr; }

}  // namespace
}  // namespace dard

using namespace dard;

extern "C" {

dard_status dard_residual_norm(const dard_norm_args* a, void* stream) {
  report(DARD_OK, "%s", "");
  if (!a) return report(DARD_ERR_NULL, "args is NULL");
  if (a->rows < 0 || a->rows > 0x7fffffffll)
    return report(DARD_ERR_SHAPE, "rows %lld outside 0..2^31 - 1", static_cast<long long>(a->rows));
  if (a->dim < 1 || a->dim > DARD_NORM_MAX_DIM)
    return report(DARD_ERR_SHAPE, "dim %d outside 1..%d", a->dim, DARD_NORM_MAX_DIM);
  if (a->dtype != DARD_BF16 && a->dtype != DARD_F32)
    return report(DARD_ERR_VALUE, "dtype %d is neither DARD_F32 nor DARD_BF16", a->dtype);
  if (!(a->eps >= 0.f) || !std::isfinite(a->eps))
    return report(DARD_ERR_VALUE, "eps must be finite and >= 0");
  if (a->y8 && a->dim % kMxBlock != 0)
    return report(DARD_ERR_SHAPE, "y8 needs dim %% 32 == 0, got %d", a->dim);
  const auto short_stride = [&](const void* p, int64_t stride) { return p && stride < a->dim; };
  if (a->x_stride < a->dim || short_stride(a->delta, a->delta_stride) ||
      short_stride(a->residual, a->residual_stride) || short_stride(a->y, a->y_stride) ||
      short_stride(a->y8, a->y8_stride) || (a->y8 && a->y8_scale_stride < a->dim / kMxBlock))
    return report(DARD_ERR_SHAPE, "a row stride is below dim (y8_scale_stride: dim / 32)");
  if (a->rows == 0) return DARD_OK;
  if (!a->x) return report(DARD_ERR_NULL, "x is NULL");
  if (!a->residual && !a->y && !a->y8)
    return report(DARD_ERR_NULL, "every output (residual, y, y8) is NULL");
  if (a->y8 && !a->y8_scale) return report(DARD_ERR_NULL, "y8 needs y8_scale");
  if (a->residual && a->residual == a->y)
    return report(DARD_ERR_VALUE, "residual and y are one buffer");
  const size_t esz = a->dtype == DARD_BF16 ? 2 : 4;
  if (!multiple(a->x, esz) || !multiple(a->delta, esz) || !multiple(a->weight, esz) ||
      !multiple(a->residual, esz) || !multiple(a->y, esz))
    return report(DARD_ERR_ALIGN, "a pointer is not a multiple of the element size");
  if (a->y8 && (a->y8_scale_stride % 16 != 0 || !multiple(a->y8_scale, 16)))
    return report(DARD_ERR_ALIGN, "y8_scale must be 16-byte aligned with a 16-byte row pitch");
  NormParams p = {};
  p.x = a->x;
  p.delta = a->delta;
  p.weight = a->weight;
  p.residual = a->residual;
  p.y = a->y;
  p.y8 = a->y8;
  p.y8_scale = a->y8_scale;
  p.rows = a->rows;
  p.x_stride = a->x_stride;
  p.delta_stride = a->delta_stride;
  p.residual_stride = a->residual_stride;
  p.y_stride = a->y_stride;
  p.y8_stride = a->y8_stride;
  p.scale_stride = a->y8_scale_stride;
  p.dim = a->dim;
  p.eps = a->eps;
  p.inv_dim = static_cast<float>(1.0 / a->dim);
  // 16-byte accesses: eight elements per run, so dim and the strides are multiples of eight
  const auto wide = [&](const void* q, int64_t stride) {
    return !q || (multiple(q, 16) && stride % 8 == 0);
  };
  const bool vec = a->dim % 8 == 0 && wide(a->x, a->x_stride) && wide(a->delta, a->delta_stride) &&
                   wide(a->weight, 0) && wide(a->residual, a->residual_stride) &&
                   wide(a->y, a->y_stride) &&
                   (!a->y8 || (multiple(a->y8, 8) && a->y8_stride % 8 == 0));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = fail_launch()              ? cudaErrorLaunchFailure
                        : a->dtype == DARD_BF16    ? launch_norm<__nv_bfloat16>(p, vec, s)
                                                   : launch_norm<float>(p, vec, s);
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "norm launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

dard_status dard_mx_quantize(const dard_mx_args* a, void* stream) {
  report(DARD_OK, "%s", "");
  if (!a) return report(DARD_ERR_NULL, "args is NULL");
  if (a->batch < 0 || a->rows < 0 || a->cols < 1 || a->cols % kMxBlock != 0)
    return report(DARD_ERR_SHAPE, "batch and rows must be >= 0, cols a positive multiple of 32");
  // (by division: the product of sizes such as these does not fit 64 bits)
  if (a->batch > 0 && a->rows > (1ll << 40) / a->cols / a->batch)
    return report(DARD_ERR_SHAPE, "more than 2^40 elements");
  if (a->dtype != DARD_BF16 && a->dtype != DARD_F32)
    return report(DARD_ERR_VALUE, "dtype %d is neither DARD_F32 nor DARD_BF16", a->dtype);
  if (a->layout != DARD_MX_SCALE_ROWS && a->layout != DARD_MX_SCALE_TILES)
    return report(DARD_ERR_VALUE, "layout %d is not a dard_mx_scale_layout", a->layout);
  if (a->x_row_stride < a->cols || a->x_batch_stride < 0)
    return report(DARD_ERR_SHAPE, "x_row_stride is below cols, or x_batch_stride below 0");
  const bool by_rows = a->layout == DARD_MX_SCALE_ROWS;
  if (by_rows && a->scale_stride < a->cols / kMxBlock)
    return report(DARD_ERR_SHAPE, "scale_stride is below cols / 32");
  if (a->batch == 0 || a->rows == 0) return DARD_OK;
  if (!a->x || !a->codes || !a->scales) return report(DARD_ERR_NULL, "x, codes or scales is NULL");
  const size_t esz = a->dtype == DARD_BF16 ? 2 : 4;
  if (!multiple(a->x, esz))
    return report(DARD_ERR_ALIGN, "x is not a multiple of the element size");
  if (!multiple(a->codes, 16) || !multiple(a->scales, 16) || (by_rows && a->scale_stride % 16 != 0))
    return report(DARD_ERR_ALIGN, "codes, scales and the scales' row pitch must be multiples of "
                                  "16 bytes");
  MxParams p = {};
  p.x = a->x;
  p.codes = a->codes;
  p.scales = a->scales;
  p.rows = a->rows;
  p.total_rows = a->batch * a->rows;
  p.x_row_stride = a->x_row_stride;
  p.x_batch_stride = a->x_batch_stride;
  p.scale_stride = a->scale_stride;
  p.cols = a->cols;
  p.tile_cols = (a->cols + 127) / 128;
  p.tiles_per_matrix = (a->rows + 127) / 128 * p.tile_cols;
  p.layout = a->layout;
  p.runs = a->cols / 16;
  // matrices that follow one another, with whole tiles of scales, are one tall matrix
  const bool follow = a->batch == 1 || a->x_batch_stride == a->rows * a->x_row_stride;
  p.one = follow && (by_rows || a->batch == 1 || a->rows % 128 == 0);
  const bool vec = multiple(a->x, 16) && a->x_row_stride % 8 == 0 && a->x_batch_stride % 8 == 0;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = fail_launch() ? cudaErrorLaunchFailure : cudaSuccess;
  if (e == cudaSuccess && !by_rows && (a->rows % 128 != 0 || a->cols % 128 != 0))
    e = cudaMemsetAsync(a->scales, 0, a->batch * p.tiles_per_matrix * kMxTileBytes, s);
  if (e == cudaSuccess)
    e = a->dtype == DARD_BF16 ? launch_mx<__nv_bfloat16>(p, vec, s) : launch_mx<float>(p, vec, s);
  if (e != cudaSuccess)
    return report(DARD_ERR_CUDA, "MXFP8 launch failed: %s", cudaGetErrorString(e));
  return DARD_OK;
}

}  // extern "C"
