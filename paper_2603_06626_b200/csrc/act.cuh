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

// Value and slope of two elements: one exponential and one reciprocal each.
template <int ACT>
__device__ __forceinline__ void act_value_slope2(float2 z, float2& value, float2& slope) {
  if (ACT == GROUTER_ACT_RELU) {
    value = make_float2(act_value<ACT>(z.x), act_value<ACT>(z.y));
    slope = make_float2(z.x > 0.f ? 1.f : 0.f, z.y > 0.f ? 1.f : 0.f);
  } else if (ACT == GROUTER_ACT_SILU) {        // s,  s + z s (1 - s)
    const float2 s = make_float2(logistic(z.x), logistic(z.y));
    value = mul2(z, s);
    slope = fma2(value, fma2(s, both(-1.f), both(1.f)), s);
  } else if (ACT == GROUTER_ACT_GELU) {        // s,  s + z s (1 - s) u',  as in act_back2
    const float2 zc = make_float2(fminf(fmaxf(z.x, -12.f), 12.f), fminf(fmaxf(z.y, -12.f), 12.f));
    const float2 q = mul2(zc, zc);
    const float2 u = mul2(zc, fma2(q, both(1.5957691216057308f * 0.044715f), both(1.5957691216057308f)));
    const float2 s = make_float2(logistic(u.x), logistic(u.y));
    value = mul2(z, s);
    slope = fma2(mul2(value, fma2(s, both(-1.f), both(1.f))), fma2(q, both(1.5957691216057308f * 0.134145f), both(1.5957691216057308f)), s);
  } else {
    value = z;
    slope = both(1.f);
  }
}
// h = act(g) u and, from h's gradient dh, dg = dh u act'(g) and du = dh act(g).
template <int ACT, int N>
__device__ __forceinline__ void gate_back(const float (&dh)[N], const float (&g)[N], const float (&u)[N], float (&h)[N], float (&dg)[N], float (&du)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const float2 d = make_float2(dh[i], dh[i + 1]), up = make_float2(u[i], u[i + 1]);
    float2 a, slope;
    act_value_slope2<ACT>(make_float2(g[i], g[i + 1]), a, slope);
    const float2 o0 = mul2(a, up), o1 = mul2(mul2(d, up), slope), o2 = mul2(d, a);
    h[i] = o0.x;
    h[i + 1] = o0.y;
    dg[i] = o1.x;
    dg[i + 1] = o1.y;
    du[i] = o2.x;
    du[i + 1] = o2.y;
  }
}

}  // namespace grouter
