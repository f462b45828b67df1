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
constexpr int FP8_MAX_COLS = 1 << 27;        // longest row (columns are counted in 32 bits, a grid's y takes 65535 x 8 atoms of 512)

__host__ __device__ inline int64_t fp8_atoms_across(int64_t cols) { return (cols + 4 * FP8_BLOCK - 1) / (4 * FP8_BLOCK); }
__host__ __device__ inline int64_t fp8_pitch(int64_t cols) { return (cols + 15) / 16 * 16; }
// Place of the scale of (row, block).
__device__ __forceinline__ int64_t fp8_scale_at(int64_t row, int block, int64_t atoms_across) {
  const int r = (int)(row & 127);
  return ((row >> 7) * atoms_across + (block >> 2)) * FP8_ATOM + (r & 31) * 16 + (r >> 5) * 4 + (block & 3);
}

// The largest magnitude is looked for among all numbers first (NaN falls out of a maximum by itself): only where it comes out infinite
// are the finite ones picked, and infinities told from 448 when codes are made.
__device__ __forceinline__ float larger(float top, float v) { return fmaxf(top, fabsf(v)); }
__device__ __forceinline__ bool not_finite(float top) { return __float_as_uint(top) >= 0x7f800000u; }
__device__ __forceinline__ float larger_finite(float top, float v) { return not_finite(fabsf(v)) ? top : larger(top, v); }

// e + 127 of the largest magnitude: its exponent less 8, one more where its mantissa is above 1.75 (448 = 1.75 * 2^8).
__device__ __forceinline__ uint32_t fp8_exponent(float top) {
  const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8;
  return e < 1 ? 1u : (uint32_t)e;
}
__device__ __forceinline__ float fp8_inverse(uint32_t exponent) { return __uint_as_float((254u - exponent) << 23); }   // 2^-e
__device__ __forceinline__ float fp8_scale(uint32_t exponent) { return __uint_as_float(exponent << 23); }              // 2^e

// Two values as codes.  INF: some may be infinite, which the conversion by itself would make 448; they become NaN.
template <bool INF>
__device__ __forceinline__ uint32_t fp8_pair(float2 v, float2 inverse) {
  v = mul2(v, inverse);
  if (INF) {
    const float nan = __uint_as_float(0x7fffffffu);
    if (not_finite(fabsf(v.x))) v.x = nan;
    if (not_finite(fabsf(v.y))) v.y = nan;
  }
  return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
}
template <bool INF>
__device__ __forceinline__ uint32_t fp8_quad(const float* v, float inverse) {
  return fp8_pair<INF>(make_float2(v[0], v[1]), both(inverse)) | fp8_pair<INF>(make_float2(v[2], v[3]), both(inverse)) << 16;
}
__device__ __forceinline__ float2 fp8_values(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Largest of the LANES neighbouring lanes' magnitudes, the same in each of them.  Bits of numbers that are not negative are in order.
template <int LANES>
__device__ __forceinline__ float lanes_top(float v) {
  if constexpr (LANES == 32) return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
  else return lanes_max<LANES>(v);
}

// ---- blocks as the quantizing kernels hold them: sixteen neighbours a lane, as they lie in memory, eight lanes a block ----
// Magnitudes in progress: of one f32 (as itself) or of two bf16 (as 16-bit halves of a word).
template <typename T>
__device__ __forceinline__ uint32_t word_top(uint32_t top, uint32_t w) {
  if constexpr (sizeof(T) == 4) return max(top, w & 0x7fffffffu);
  else return __vmaxu2(top, w & 0x7fff7fffu);
}
// ... without what is not finite
template <typename T>
__device__ __forceinline__ uint32_t word_top_finite(uint32_t top, uint32_t w) {
  if constexpr (sizeof(T) == 4) {
    w &= 0x7fffffffu;
    return w < 0x7f800000u ? max(top, w) : top;
  } else {
    w &= 0x7fff7fffu;
    if ((w & 0xffffu) >= 0x7f80u) w &= 0xffff0000u;
    if (w >= 0x7f800000u) w &= 0xffffu;
    return __vmaxu2(top, w);
  }
}
// the larger half of a pair, as the bits of an f32
template <typename T>
__device__ __forceinline__ uint32_t top_of_word(uint32_t top) {
  if constexpr (sizeof(T) == 4) return top;
  else return max(top << 16, top & 0xffff0000u);
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_top_bits(uint32_t v) {
  if constexpr (LANES == 32) return __reduce_max_sync(0xffffffffu, v);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ bool bits_not_finite(uint32_t top) { return top >= 0x7f800000u; }
// Elements 2j and 2j + 1 of some words, as f32.
template <typename T>
__device__ __forceinline__ float2 word_pair(const uint32_t* w, int j) {
  if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
  else return make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
}

constexpr int Q_LANE = 16;                // neighbours a lane takes
constexpr int Q_LANES = FP8_BLOCK / Q_LANE;      // lanes that hold a block
template <typename T>
__host__ __device__ constexpr int q_words() { return Q_LANE * (int)sizeof(T) / 4; }

template <typename T>
__device__ __forceinline__ uint32_t lane_top(const uint32_t (&w)[q_words<T>()]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < q_words<T>(); ++i) top = word_top<T>(top, w[i]);
  return top_of_word<T>(top);
}
template <typename T>
__device__ __forceinline__ uint32_t lane_top_finite(const uint32_t (&w)[q_words<T>()]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < q_words<T>(); ++i) top = word_top_finite<T>(top, w[i]);
  return top_of_word<T>(top);
}
// Exponent + 127 of the block that Q_LANES neighbouring lanes hold; inf: some element of the warp is not finite.
template <typename T>
__device__ __forceinline__ uint32_t block_exponent(const uint32_t (&w)[q_words<T>()], bool& inf) {
  uint32_t top = lanes_top_bits<Q_LANES>(lane_top<T>(w));
  inf = __any_sync(0xffffffffu, bits_not_finite(top));
  if (inf) top = lanes_top_bits<Q_LANES>(lane_top_finite<T>(w));
  return fp8_exponent(__uint_as_float(top));
}
// The same of two rows' blocks at once: two bf16 maxima are halves of a word, so that the lanes compare both with one shuffle.
template <typename T>
__device__ __forceinline__ void block_exponents(const uint32_t (&w)[2][q_words<T>()], uint32_t (&e)[2], bool& inf) {
  if constexpr (sizeof(T) == 4) {
    bool inf1;
    e[0] = block_exponent<T>(w[0], inf);
    e[1] = block_exponent<T>(w[1], inf1);
    inf = inf || inf1;
  } else {
    uint32_t top[2] = {0, 0};
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int i = 0; i < q_words<T>(); ++i) top[r] = word_top<T>(top[r], w[r][i]);
    uint32_t t = __vmaxu2(__byte_perm(top[0], top[1], 0x5410), __byte_perm(top[0], top[1], 0x7632));
#pragma unroll
    for (int o = Q_LANES / 2; o > 0; o >>= 1) t = __vmaxu2(t, __shfl_xor_sync(0xffffffffu, t, o));
    uint32_t bits[2] = {t << 16, t & 0xffff0000u};
    inf = __any_sync(0xffffffffu, bits_not_finite(bits[0]) || bits_not_finite(bits[1]));
    if (inf) {
#pragma unroll
      for (int r = 0; r < 2; ++r) bits[r] = lanes_top_bits<Q_LANES>(lane_top_finite<T>(w[r]));
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) e[r] = fp8_exponent(__uint_as_float(bits[r]));
  }
}
template <typename T, bool INF>
__device__ __forceinline__ uint4 lane_codes(const uint32_t (&w)[q_words<T>()], float2 inv) {
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = fp8_pair<INF>(word_pair<T>(w, 2 * i), inv) | fp8_pair<INF>(word_pair<T>(w, 2 * i + 1), inv) << 16;
  return make_uint4(q[0], q[1], q[2], q[3]);
}

}  // namespace grouter
