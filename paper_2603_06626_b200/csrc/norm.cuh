// Pieces of the kernels that normalise the rows of a matrix: weights, sums over a row's threads, columns' sums.
#pragma once
#include "vec.cuh"

namespace grouter {

// VE consecutive weights from column c on (which exist), as f32.
template <typename W, int VE>
__device__ __forceinline__ void load_weights(const W* __restrict__ w, int c, float (&f)[VE]) {
  if constexpr (VE == 1) {
    f[0] = to_f32(__ldg(w + c));
  } else {
    constexpr int PER = VE * sizeof(W) >= 16 ? 16 / (int)sizeof(W) : VE;       // accesses of 16, 8 or 4 bytes
#pragma unroll
    for (int q = 0; q < VE; q += PER) {
      Pack<W, PER> p;
      if constexpr (PER * sizeof(W) == 16) *reinterpret_cast<uint4*>(&p) = __ldg(reinterpret_cast<const uint4*>(w + c + q));
      else if constexpr (PER * sizeof(W) == 8) *reinterpret_cast<uint2*>(&p) = __ldg(reinterpret_cast<const uint2*>(w + c + q));
      else *reinterpret_cast<uint32_t*>(&p) = __ldg(reinterpret_cast<const uint32_t*>(w + c + q));
      const Pack<W, PER> one[1] = {p};
#pragma unroll
      for (int i = 0; i < PER; i += 2) {
        const float2 v = pair_at(one, i / 2);
        f[q + i] = v.x;
        f[q + i + 1] = v.y;
      }
    }
  }
}

// Sums of N values over the LANES threads of a row, the same value in each of them.  `red` has two halves used in turn: a warp
// may still read one while the others already write the next sums into the other, and the barrier in between keeps the third away.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& half) {
  constexpr int NW = LANES / 32;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lanes_sum<(LANES < 32 ? LANES : 32)>(v[n]);
  if constexpr (NW > 1) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* buf = red + half * (N * 32);
    half ^= 1;
    if (lane == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) buf[n * 32 + warp] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<NW>(buf[n * 32 + (lane & (NW - 1))]);
  }
}

// Nothing about these registers is known from here on: the compiler converts them again where they are used next, instead of
// carrying twice as many converted values along.
template <typename T, int VE, int NP>
__device__ __forceinline__ void forget(Pack<T, VE> (&p)[NP]) {
  if constexpr (VE > 1 && sizeof(T) == 2) {
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      uint32_t* r = reinterpret_cast<uint32_t*>(&p[n]);
#pragma unroll
      for (int i = 0; i < VE / 2; ++i) asm volatile("" : "+r"(r[i]));
    }
  }
}

// VE floats at(0), at(1), ... to consecutive places, 16 bytes at a time where there are four or more (whose place is a multiple of them).
template <int VE, typename At>
__device__ __forceinline__ void store_floats(float* to, At at) {
  if constexpr (VE == 1) {
    to[0] = at(0);
  } else if constexpr (VE == 2) {
    *reinterpret_cast<float2*>(to) = make_float2(at(0), at(1));
  } else {
#pragma unroll
    for (int i = 0; i < VE; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(at(i), at(i + 1), at(i + 2), at(i + 3));
  }
}

}  // namespace grouter
