// AdamW (decoupled weight decay) over a list of tensors in one launch, moments in 32 or in 8 bits.
//
//   g' = s g                       (s: optional scale on the device, e.g. a clipping coefficient)
//   m  = b1 m + (1 - b1) g'        v = b2 v + (1 - b2) g'^2
//   p  = p (1 - lr wd) - (lr / c1) m / (sqrt(v) / sqrt(c2) + eps)          c1 = 1 - b1^t, c2 = 1 - b2^t
//
// Parameters are f32 (updated in place) or bf16 with an f32 master copy that is updated and rounded into them.  The moments
// (and the masters) of all tensors lie in flat buffers, every tensor from a multiple of 32 elements on.
//
// 8-bit moments: 32 consecutive elements share a power-of-two scale 2^x (one byte, x + 127), the smallest one under which
// their largest magnitude is at most 448; each is kept as an e4m3 code of value / 2^x, rounded to nearest even.  Kept are m
// and sqrt(v): the root has half of v's range in octaves, which is what 4 exponent bits can carry.  A root that is there
// never rounds to zero (its code is at least the smallest one): a kept m over a lost root would make a step of m / eps.
// The step itself uses the new moments before they are rounded.
//
// Every product, sum, quotient and root is rounded separately (no contraction), in the order written above: the result of
// an element does not depend on which code path or compiler handles it.
// Bound by HBM: 30 bytes an element (f32 moments and gradient, bf16 parameter), 16.06 with 8-bit moments and bf16 gradient.
// A table in device memory, built once on the host, cuts the tensors into chunks of ADAMW_CHUNK elements, one block each.
#include <cuda_fp8.h>
#include <math.h>

#include "vec.cuh"

namespace grouter {

constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_ITERS = 8;
constexpr int ADAMW_CHUNK = ADAMW_THREADS * 4 * ADAMW_ITERS;
constexpr int ADAMW_GROUP = 32;        // elements that share a scale
constexpr int P_BF16 = 1, G_BF16 = 2, P_VEC = 4, G_VEC = 8;

struct AdamwEntry {
  void* p;
  const void* g;
  int64_t n;
  int64_t offset;       // of its moments (and master) in the flat buffers, a multiple of 32
  double decay;
  int32_t flags;
  int32_t pad;
};
struct AdamwChunk {
  int32_t tensor;
  int32_t chunk;        // of that tensor
};

struct AdamwParams {
  const AdamwEntry* entries;
  const AdamwChunk* chunks;
  float* master;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  float b1, nb1, b2, nb2, inv_sqrt_c2, eps, lr_c1;
  double lr;
  const float* scale;
};

__device__ __forceinline__ float2 e4m3x2_to_f32(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3);
  return __half22float2(__half2(h));
}
__device__ __forceinline__ float pow2(int x) { return __int_as_float((x + 127) << 23); }      // -126 <= x <= 127

// Four consecutive elements of f32 or bf16; the first `n` of them exist.
__device__ __forceinline__ void load4(const void* base, bool bf16, bool vec, int64_t i, int n, float (&f)[4]) {
  if (n >= 4 && vec) {
    if (bf16) {
      const uint2 r = __ldcs(reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(base) + i));
      const float2 lo = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r.x));
      const float2 hi = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r.y));
      f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
    } else {
      const float4 r = __ldcs(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + i));
      f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w;
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[q] = 0.f;
    if (q < n) f[q] = bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(base)[i + q]) : reinterpret_cast<const float*>(base)[i + q];
  }
}
__device__ __forceinline__ void store4(void* base, bool bf16, bool vec, int64_t i, int n, const float (&f)[4]) {
  if (n >= 4 && vec) {
    if (bf16) {
      uint2 r;
      *reinterpret_cast<__nv_bfloat162*>(&r.x) = __floats2bfloat162_rn(f[0], f[1]);
      *reinterpret_cast<__nv_bfloat162*>(&r.y) = __floats2bfloat162_rn(f[2], f[3]);
      __stcs(reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(base) + i), r);
    } else {
      __stcs(reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + i), make_float4(f[0], f[1], f[2], f[3]));
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < n) {
      if (bf16) reinterpret_cast<__nv_bfloat16*>(base)[i + q] = __float2bfloat16_rn(f[q]);
      else reinterpret_cast<float*>(base)[i + q] = f[q];
    }
}

// Codes of four elements and their group's exponent byte; the eight lanes of a group call it together.  An infinite value
// becomes NaN, the one code that says "not finite".
template <bool ROOT>
__device__ __forceinline__ uint32_t encode4(const float (&f)[4], uint8_t& exp_byte) {
  float top = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const uint32_t bits = __float_as_uint(top);
  int x = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);      // top <= 1.75 * 2^8 * 2^x
  x = x < -126 ? -126 : x > 126 ? 126 : x;
  const float inv = pow2(-x);
  uint32_t code = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float2 a = make_float2(f[2 * h] * inv, f[2 * h + 1] * inv);       // exact: a power of two
    if (fabsf(a.x) == INFINITY) a.x = NAN;
    if (fabsf(a.y) == INFINITY) a.y = NAN;
    uint32_t c = __nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3);
    if (ROOT) {
      if ((c & 0xffu) == 0 && f[2 * h] > 0.f) c |= 1u;
      if ((c & 0xff00u) == 0 && f[2 * h + 1] > 0.f) c |= 0x100u;
    }
    code |= c << (16 * h);
  }
  exp_byte = (uint8_t)(x + 127);
  return code;
}
__device__ __forceinline__ void decode4(uint32_t code, uint8_t exp_byte, float (&f)[4]) {
  const float scale = pow2((int)exp_byte - 127);
  const float2 lo = e4m3x2_to_f32(code), hi = e4m3x2_to_f32(code >> 16);
  f[0] = lo.x * scale; f[1] = lo.y * scale; f[2] = hi.x * scale; f[3] = hi.y * scale;
}

template <int BITS>
__global__ void __launch_bounds__(ADAMW_THREADS) adamw_kernel(const AdamwParams a) {
  const AdamwChunk ch = a.chunks[blockIdx.x];
  const AdamwEntry en = a.entries[ch.tensor];
  const bool p_bf16 = en.flags & P_BF16, g_bf16 = en.flags & G_BF16, p_vec = en.flags & P_VEC, g_vec = en.flags & G_VEC;
  const float keep = (float)(1.0 - a.lr * en.decay);
  const float scale = a.scale ? __ldg(a.scale) : 1.f;
  const int64_t first = (int64_t)ch.chunk * ADAMW_CHUNK;
  const int64_t padded = (en.n + ADAMW_GROUP - 1) / ADAMW_GROUP * ADAMW_GROUP;      // whole groups: their lanes stay together
#pragma unroll 2
  for (int it = 0; it < ADAMW_ITERS; ++it) {
    const int64_t i = first + (int64_t)(it * ADAMW_THREADS + threadIdx.x) * 4;
    if (first + (int64_t)(it * ADAMW_THREADS) * 4 >= en.n) break;                    // the whole block is past the end
    const bool in_group = i < padded;
    const int n = !in_group || i >= en.n ? 0 : en.n - i >= 4 ? 4 : (int)(en.n - i);
    const int64_t at = en.offset + i;
    float g[4], p[4], m[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    load4(en.g, g_bf16, g_vec, i, n, g);
    if (p_bf16) load4(a.master, false, true, at, n, p);
    else load4(en.p, false, p_vec, i, n, p);
    if (in_group) {
      if constexpr (BITS == 32) {
        const float4 m4 = __ldcs(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.m) + at));
        const float4 v4 = __ldcs(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.v) + at));
        m[0] = m4.x; m[1] = m4.y; m[2] = m4.z; m[3] = m4.w;
        v[0] = v4.x; v[1] = v4.y; v[2] = v4.z; v[3] = v4.w;
      } else {
        decode4(__ldcs(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(a.m) + at)), a.m_exp[at / ADAMW_GROUP], m);
        decode4(__ldcs(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(a.v) + at)), a.v_exp[at / ADAMW_GROUP], v);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = __fmul_rn(v[q], v[q]);
      }
    }
    float root[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float gs = a.scale ? __fmul_rn(g[q], scale) : g[q];
      m[q] = __fadd_rn(__fmul_rn(m[q], a.b1), __fmul_rn(gs, a.nb1));
      v[q] = __fadd_rn(__fmul_rn(v[q], a.b2), __fmul_rn(__fmul_rn(gs, gs), a.nb2));
      root[q] = __fsqrt_rn(v[q]);
      const float den = __fadd_rn(__fmul_rn(root[q], a.inv_sqrt_c2), a.eps);
      p[q] = __fsub_rn(__fmul_rn(p[q], keep), __fmul_rn(__fdiv_rn(m[q], den), a.lr_c1));
    }
    if (p_bf16) {
      store4(a.master, false, true, at, n, p);
      store4(en.p, true, p_vec, i, n, p);
    } else {
      store4(en.p, false, p_vec, i, n, p);
    }
    if constexpr (BITS == 32) {
      if (in_group) {
        store4(a.m, false, true, at, n, m);
        store4(a.v, false, true, at, n, v);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q >= n) m[q] = root[q] = 0.f;          // the rest of the last group holds nothing
      uint8_t mx, rx;
      const uint32_t mc = encode4<false>(m, mx), rc = encode4<true>(root, rx);
      if (in_group) {
        __stcs(reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(a.m) + at), mc);
        __stcs(reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(a.v) + at), rc);
        if ((threadIdx.x & 7) == 0) {
          a.m_exp[at / ADAMW_GROUP] = mx;
          a.v_exp[at / ADAMW_GROUP] = rx;
        }
      }
    }
  }
}

// The values that 8-bit moments stand for: m_out = m, v_out = root^2.
__global__ void __launch_bounds__(256) adamw_moments_kernel(const uint8_t* __restrict__ m, const uint8_t* __restrict__ r,
                                                            const uint8_t* __restrict__ m_exp, const uint8_t* __restrict__ r_exp, int64_t n4,
                                                            float* __restrict__ m_out, float* __restrict__ v_out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    float f[4];
    decode4(__ldcs(reinterpret_cast<const uint32_t*>(m) + i), m_exp[i / 8], f);
    __stcs(reinterpret_cast<float4*>(m_out) + i, make_float4(f[0], f[1], f[2], f[3]));
    decode4(__ldcs(reinterpret_cast<const uint32_t*>(r) + i), r_exp[i / 8], f);
    __stcs(reinterpret_cast<float4*>(v_out) + i, make_float4(f[0] * f[0], f[1] * f[1], f[2] * f[2], f[3] * f[3]));
  }
}

}  // namespace grouter

using namespace grouter;

extern "C" {

int grouter_adamw_layout_host(const grouter_adamw_tensor* tensors, int32_t n_tensors, grouter_adamw_layout* layout, void* table_host) {
  if (!layout || n_tensors < 1 || !tensors) return GROUTER_ERR_INVALID_ARG;
  int64_t chunks = 0, elements = 0;
  int32_t needs_master = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const grouter_adamw_tensor& t = tensors[i];
    if (t.n < 0 || (t.n > 0 && (!t.param || !t.grad)) || !isfinite(t.weight_decay)) return GROUTER_ERR_INVALID_ARG;
    if ((t.param_dtype != GROUTER_BF16 && t.param_dtype != GROUTER_F32) || (t.grad_dtype != GROUTER_BF16 && t.grad_dtype != GROUTER_F32))
      return GROUTER_ERR_INVALID_ARG;
    if (t.n > (int64_t)1 << 40) return GROUTER_ERR_UNSUPPORTED;
    if (!aligned_to(t.param, t.param_dtype == GROUTER_BF16 ? 2 : 4) || !aligned_to(t.grad, t.grad_dtype == GROUTER_BF16 ? 2 : 4))
      return GROUTER_ERR_MISALIGNED;
    chunks += (t.n + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
    elements += (t.n + ADAMW_GROUP - 1) / ADAMW_GROUP * ADAMW_GROUP;
    if (t.param_dtype == GROUTER_BF16) needs_master = 1;
  }
  if (chunks > INT32_MAX) return GROUTER_ERR_UNSUPPORTED;
  layout->n_tensors = n_tensors;
  layout->n_chunks = (int32_t)chunks;
  layout->state_elements = elements;
  layout->table_bytes = sizeof(AdamwEntry) * (size_t)n_tensors + sizeof(AdamwChunk) * (size_t)chunks;
  layout->needs_master = needs_master;
  layout->reserved = 0;
  if (!table_host) return GROUTER_OK;
  if (!aligned_to(table_host, 8)) return GROUTER_ERR_MISALIGNED;
  AdamwEntry* e = static_cast<AdamwEntry*>(table_host);
  AdamwChunk* c = reinterpret_cast<AdamwChunk*>(e + n_tensors);
  int64_t at = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const grouter_adamw_tensor& t = tensors[i];
    const bool pb = t.param_dtype == GROUTER_BF16, gb = t.grad_dtype == GROUTER_BF16;
    e[i].p = t.param;
    e[i].g = t.grad;
    e[i].n = t.n;
    e[i].offset = at;
    e[i].decay = t.weight_decay;
    e[i].flags = (pb ? P_BF16 : 0) | (gb ? G_BF16 : 0) | (aligned_to(t.param, pb ? 8 : 16) ? P_VEC : 0) | (aligned_to(t.grad, gb ? 8 : 16) ? G_VEC : 0);
    e[i].pad = 0;
    at += (t.n + ADAMW_GROUP - 1) / ADAMW_GROUP * ADAMW_GROUP;
    for (int64_t q = 0; q * ADAMW_CHUNK < t.n; ++q, ++c) {
      c->tensor = i;
      c->chunk = (int32_t)q;
    }
  }
  return GROUTER_OK;
}

int grouter_adamw_step(const grouter_adamw_layout* layout, const void* table, int32_t state_bits, float* master, void* m, void* v,
                       uint8_t* m_exp, uint8_t* v_exp, double lr, double beta1, double beta2, double eps, int64_t step, const float* grad_scale,
                       void* stream) {
  if (!layout || layout->n_tensors < 1 || layout->n_chunks < 0 || (state_bits != 32 && state_bits != 8) || step < 1) return GROUTER_ERR_INVALID_ARG;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !isfinite(eps) || !isfinite(lr)) return GROUTER_ERR_INVALID_ARG;
  if (layout->n_chunks == 0) return GROUTER_OK;
  if (!table || !m || !v || (layout->needs_master && !master) || (state_bits == 8 && (!m_exp || !v_exp))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(table, 16) || !aligned_to(master, 16) || !aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(grad_scale, 4))
    return GROUTER_ERR_MISALIGNED;
  AdamwParams a{};
  a.entries = static_cast<const AdamwEntry*>(table);
  a.chunks = reinterpret_cast<const AdamwChunk*>(a.entries + layout->n_tensors);
  a.master = master; a.m = m; a.v = v; a.m_exp = m_exp; a.v_exp = v_exp;
  const double c1 = 1.0 - pow(beta1, (double)step), c2 = 1.0 - pow(beta2, (double)step);
  a.b1 = (float)beta1;
  a.nb1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.nb2 = (float)(1.0 - beta2);
  a.inv_sqrt_c2 = (float)(1.0 / sqrt(c2));
  a.eps = (float)eps;
  a.lr_c1 = (float)(lr / c1);
  a.lr = lr;
  a.scale = grad_scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (state_bits == 32) adamw_kernel<32><<<layout->n_chunks, ADAMW_THREADS, 0, st>>>(a);
  else adamw_kernel<8><<<layout->n_chunks, ADAMW_THREADS, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

int grouter_adamw_moments(const void* m, const void* v, const uint8_t* m_exp, const uint8_t* v_exp, int64_t elements, float* m_out, float* v_out,
                          void* stream) {
  if (elements < 0 || elements % ADAMW_GROUP) return GROUTER_ERR_INVALID_ARG;
  if (elements == 0) return GROUTER_OK;
  if (!m || !v || !m_exp || !v_exp || !m_out || !v_out) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(m_out, 16) || !aligned_to(v_out, 16)) return GROUTER_ERR_MISALIGNED;
  const int64_t n4 = elements / 4, want = (n4 + 255) / 256, cap = (int64_t)current_sms() * 16;
  adamw_moments_kernel<<<(int)(want < cap ? want : cap), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint8_t*>(m), static_cast<const uint8_t*>(v), m_exp, v_exp, n4, m_out, v_out);
  return cudaGetLastError() == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
