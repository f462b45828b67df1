// Matrices in 8 bits: e4m3 codes [rows, pitch] and one power-of-two scale for 128 neighbours of a row.
//
//   scale 2^e: the smallest with |v| <= 448 * 2^e for every finite v of the block, -126 <= e      (448: the largest e4m3 number)
//   code  v * 2^-e (exact) rounded to nearest even; what is not finite has the NaN code and no say in the scale
//
// Powers of two, because the tensor cores multiply by them on the way (block scaling takes 8-bit exponents): the scales cost the
// product nothing, and quantizing is exact but for the one rounding.  A code keeps its 3 bits of mantissa whatever the scale, so a
// free scale would gain only where codes get subnormal, some 2^-14 of the largest and below.
// Scales are kept in the order in which the tensor cores take them: 512 bytes ("atom") for 128 rows and four blocks of a row, atoms
// [rows / 128][blocks / 4], in them the byte of row r, block b at (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4.  The bytes of rows and
// blocks that are not there hold anything.
#pragma once
#include <cuda_fp8.h>

#include "vec.cuh"

namespace grouter {

constexpr int FP8_BLOCK = 128;
constexpr int FP8_ATOM = 512;

__host__ __device__ inline int64_t fp8_atoms_across(int64_t cols) { return (cols + 4 * FP8_BLOCK - 1) / (4 * FP8_BLOCK); }
__host__ __device__ inline int64_t fp8_pitch(int64_t cols) { return (cols + 15) / 16 * 16; }
// Place of the scale of (row, block).
__device__ __forceinline__ int64_t fp8_scale_at(int64_t row, int block, int64_t atoms_across) {
  const int r = (int)(row & 127);
  return ((row >> 7) * atoms_across + (block >> 2)) * FP8_ATOM + (r & 31) * 16 + (r >> 5) * 4 + (block & 3);
}

// Magnitude as bits, in which finite numbers are ordered; 0 for what is not finite.
__device__ __forceinline__ uint32_t finite_magnitude(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// e + 127 from the bits of the largest magnitude: its exponent less 8, one more where its mantissa is above 1.75 (448 = 1.75 * 2^8).
__device__ __forceinline__ uint32_t fp8_exponent(uint32_t top) {
  const int e = (int)((top + 0x1fffffu) >> 23) - 8;
  return e < 1 ? 1u : (uint32_t)e;
}
__device__ __forceinline__ float fp8_inverse(uint32_t exponent) { return __uint_as_float((254u - exponent) << 23); }   // 2^-e
__device__ __forceinline__ float fp8_scale(uint32_t exponent) { return __uint_as_float(exponent << 23); }              // 2^e

// Two values, already divided by the scale, as codes; infinities (which the conversion would make 448) as NaN.
__device__ __forceinline__ uint32_t fp8_pair(float a, float b) {
  const float inf = __uint_as_float(0x7f800000u), nan = __uint_as_float(0x7fffffffu);
  if (fabsf(a) == inf) a = nan;
  if (fabsf(b) == inf) b = nan;
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t fp8_quad(const float* v, float inverse) {
  return fp8_pair(v[0] * inverse, v[1] * inverse) | fp8_pair(v[2] * inverse, v[3] * inverse) << 16;
}
__device__ __forceinline__ float2 fp8_values(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

template <int LANES>
__device__ __forceinline__ uint32_t lanes_max_bits(uint32_t v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

}  // namespace grouter
