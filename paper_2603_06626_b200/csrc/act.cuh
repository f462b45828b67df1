// Activations of the linear layer and their slopes.
#pragma once
#include "common.cuh"

namespace grouter {

// 1 / (1 + exp(-z)) with the hardware's exponential and reciprocal (each within 2 ulp); where exp overflows it is 0.
__device__ __forceinline__ float logistic(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}

// GELU in its tanh form is z times a logistic:  (1 + tanh u) / 2 = logistic(2u),  u = sqrt(2/pi) (z + 0.044715 z^3).
// Beyond |z| = 12 the logistic is 0 or 1 in fp32, so the cubic is evaluated on z clamped there and cannot overflow.
__device__ __forceinline__ float gelu_gate(float z, float& zc) {
  zc = fminf(fmaxf(z, -12.f), 12.f);
  return logistic(1.5957691216057308f * (zc + 0.044715f * zc * zc * zc));
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == GROUTER_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (ACT == GROUTER_ACT_SILU) return z * logistic(z);
  if (ACT == GROUTER_ACT_GELU) {
    float zc;
    return z * gelu_gate(z, zc);
  }
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == GROUTER_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == GROUTER_ACT_SILU) {
    const float s = logistic(z);
    return s * (1.f + z * (1.f - s));
  }
  if (ACT == GROUTER_ACT_GELU) {
    float zc;
    const float s = gelu_gate(z, zc);
    return s + z * s * (1.f - s) * 1.5957691216057308f * (1.f + 0.134145f * zc * zc);
  }
  return 1.f;
}

}  // namespace grouter
