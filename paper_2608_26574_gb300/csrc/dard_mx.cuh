// dard_mx.cuh - device pieces of the MXFP8 rounding (include/dard.h): the scale byte of a
// block from its largest magnitude, and the e4m3 codes.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

namespace dard {

constexpr int kMxBlock = 32;      // elements per scale
constexpr int kMxTileBytes = 512; // scales of 128 rows x 4 blocks (128 elements)

// Byte of row r, block c within its 128 x 4 tile of scales.
__host__ __device__ constexpr int mx_tile_byte(int r, int c) {
  return (r % 32) * 16 + (r % 128) / 32 * 4 + c % 4;
}

// Maximum that keeps a NaN of either operand (fmaxf drops it).
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// The scale byte of a block with largest magnitude `amax` (NaN if the block holds one): with
// amax = m 2^x, 1 <= m < 2, the smallest e with amax 2^-e <= 448 = 1.75 * 2^8 is x - 8 for
// m <= 1.75 and x - 7 above. Exact: both are read from the bits.
__device__ __forceinline__ uint32_t mx_scale_byte(float amax) {
  const uint32_t bits = __float_as_uint(amax) & 0x7fffffffu;
  if (bits >= 0x7f800000u) return 255u;  // a NaN or an infinity in the block
  const int b = static_cast<int>(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(max(b, 0));
}

// 2^(127 - byte), by which a block is multiplied before rounding; NaN for byte 255. (The
// largest byte of a finite block is 247, so the exponent field stays within 7 .. 254.)
__device__ __forceinline__ float mx_inverse(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7fc00000u : (254u - byte) << 23);
}

// Two e4m3 codes (nearest, ties to even): lo in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}

}  // namespace dard
