// Activations of the linear layer and their slopes.
#pragma once
#include "vec.cuh"

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
// g times the slope at z, two elements at a time.
template <int ACT>
__device__ __forceinline__ float2 act_back2(float2 g, float2 z) {
  if (ACT == GROUTER_ACT_RELU) return make_float2(z.x > 0.f ? g.x : 0.f, z.y > 0.f ? g.y : 0.f);
  if (ACT == GROUTER_ACT_SILU) {        // s (1 + z (1 - s))
    const float2 s = make_float2(logistic(z.x), logistic(z.y));
    const float2 rest = fma2(s, both(-1.f), both(1.f));
    return mul2(g, mul2(s, fma2(z, rest, both(1.f))));
  }
  if (ACT == GROUTER_ACT_GELU) {        // s + z s (1 - s) u',  u' = 2 sqrt(2/pi) (1 + 3 * 0.044715 z^2)
    const float2 zc = make_float2(fminf(fmaxf(z.x, -12.f), 12.f), fminf(fmaxf(z.y, -12.f), 12.f));
    const float2 q = mul2(zc, zc);
    const float2 u = mul2(zc, fma2(q, both(1.5957691216057308f * 0.044715f), both(1.5957691216057308f)));
    const float2 s = make_float2(logistic(u.x), logistic(u.y));
    const float2 slope = fma2(q, both(1.5957691216057308f * 0.134145f), both(1.5957691216057308f));
    const float2 rest = fma2(s, both(-1.f), both(1.f));
    return mul2(g, fma2(mul2(mul2(z, s), rest), slope, s));
  }
  return g;
}

// v = act(v) for an activation that is known at run time only.
template <int N>
__device__ __forceinline__ void act_values(float (&v)[N], int act) {
  if (act == GROUTER_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<GROUTER_ACT_RELU>(v[i]);
  } else if (act == GROUTER_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<GROUTER_ACT_SILU>(v[i]);
  } else if (act == GROUTER_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<GROUTER_ACT_GELU>(v[i]);
  }
}

// Backward of act(g) u from its gradient dg: a = act(g), and dg becomes the gate's, dg u act'(g).
template <int ACT, int N>
__device__ __forceinline__ void act_gate_back(float (&dg)[N], const float (&g)[N], const float (&u)[N], float (&a)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const float2 d = act_back2<ACT>(mul2(make_float2(dg[i], dg[i + 1]), make_float2(u[i], u[i + 1])), make_float2(g[i], g[i + 1]));
    dg[i] = d.x;
    dg[i + 1] = d.y;
    a[i] = act_value<ACT>(g[i]);
    a[i + 1] = act_value<ACT>(g[i + 1]);
  }
}
template <int N>
__device__ __forceinline__ void act_gate_backward(float (&dg)[N], const float (&g)[N], const float (&u)[N], float (&a)[N], int act) {
  if (act == GROUTER_ACT_RELU) act_gate_back<GROUTER_ACT_RELU, N>(dg, g, u, a);
  else if (act == GROUTER_ACT_SILU) act_gate_back<GROUTER_ACT_SILU, N>(dg, g, u, a);
  else if (act == GROUTER_ACT_GELU) act_gate_back<GROUTER_ACT_GELU, N>(dg, g, u, a);
  else act_gate_back<GROUTER_ACT_NONE, N>(dg, g, u, a);
}

}  // namespace grouter
