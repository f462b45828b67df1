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
// Bound by HBM: 30 bytes an element (f32 moments and gradient, bf16 parameter), 16.125 with 8-bit moments and bf16 gradient.
// Measured: 138 M elements with f32 moments 605-615 us (6.8 TB/s, a little above a plain copy's 6.46: reads outweigh writes);
// 69 M with 8-bit moments and bf16 gradient 200 us (5.5 TB/s), 6 M of them in 120 tensors 21 us and 10 us to read the moments back.
// The 8-bit form spends some 60 instructions an element, most of them on the exactly rounded root and quotient and on the codes:
// whole chunks go without any test, two groups' exponents are reduced in one word, what is rare (values below the smallest code,
// infinities) is behind a branch (and 8 bytes a thread are spilled, at five blocks an SM).
// A table in device memory, built once on the host, cuts the tensors into chunks of ADAMW_CHUNK elements, one block each: small, so
// that an SM always has blocks that load while others compute (8192 elements a block: 35 against 31 us for 6 M elements in
// 120 small tensors with 8-bit moments, 620 against 604 us for 138 M with f32 moments).
#include <cuda_fp8.h>
#include <math.h>

#include <algorithm>
#include <memory>
#include <new>

#include "vec.cuh"

namespace grouter {

constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_CHUNK = ADAMW_THREADS * 8;     // one step of the 8-bit form, two of the other
constexpr int ADAMW_GROUP = 32;        // elements that share a scale
constexpr int P_BF16 = 1, G_BF16 = 2, P_VEC = 4, G_VEC = 8;

// One block's work: up to ADAMW_CHUNK elements of one tensor.  Everything it needs to know is here, one load away.
struct AdamwChunk {
  void* p;              // its first parameter and gradient
  const void* g;
  int64_t flat;         // its first moment (and master) in the flat buffers, a multiple of 32
  double decay;
  int32_t n;
  int32_t flags;
};

struct AdamwParams {
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

// Four consecutive elements of f32 or bf16 as they lie in memory; the first n of them exist (the others read as zero).  FULL: all
// of them, and base lies on the boundary that a whole access needs.
template <bool HALF>
struct Four {
  uint32_t w[HALF ? 2 : 4];
};
template <bool HALF, bool FULL>
__device__ __forceinline__ Four<HALF> load4(const void* base, bool vec, int n) {
  Four<HALF> r;
  if (FULL || (n >= 4 && vec)) {
    if constexpr (HALF) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(base));
      r.w[0] = v.x; r.w[1] = v.y;
    } else {
      const uint4 v = __ldcs(reinterpret_cast<const uint4*>(base));
      r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    }
    return r;
  }
  if constexpr (FULL) {
  } else if constexpr (HALF) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(base);
    r.w[0] = (n > 0 ? p[0] : 0u) | (n > 1 ? (uint32_t)p[1] << 16 : 0u);
    r.w[1] = (n > 2 ? p[2] : 0u) | (n > 3 ? (uint32_t)p[3] << 16 : 0u);
  } else {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(base);
#pragma unroll
    for (int q = 0; q < 4; ++q) r.w[q] = q < n ? p[q] : 0u;
  }
  return r;
}
template <bool HALF>
__device__ __forceinline__ void open4(const Four<HALF>& r, float* f) {
  if constexpr (HALF) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f[2 * h] = __uint_as_float(r.w[h] << 16);
      f[2 * h + 1] = __uint_as_float(r.w[h] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] = __uint_as_float(r.w[q]);
  }
}
template <bool HALF, bool FULL>
__device__ __forceinline__ void store4(void* base, bool vec, int n, const float* f) {
  if (FULL || (n >= 4 && vec)) {
    if constexpr (HALF) {
      uint2 r;
      *reinterpret_cast<__nv_bfloat162*>(&r.x) = __floats2bfloat162_rn(f[0], f[1]);
      *reinterpret_cast<__nv_bfloat162*>(&r.y) = __floats2bfloat162_rn(f[2], f[3]);
      __stcs(reinterpret_cast<uint2*>(base), r);
    } else {
      __stcs(reinterpret_cast<float4*>(base), make_float4(f[0], f[1], f[2], f[3]));
    }
    return;
  }
  if constexpr (!FULL) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < n) {
        if constexpr (HALF) reinterpret_cast<__nv_bfloat16*>(base)[q] = __float2bfloat16_rn(f[q]);
        else reinterpret_cast<float*>(base)[q] = f[q];
      }
  }
}

// The update of one element; m, v and p become the new ones, the root of v is returned.
__device__ __forceinline__ float adamw_element(const AdamwParams& a, float scale, float keep, float g, float& p, float& m, float& v) {
  const float gs = __fmul_rn(g, scale);                     // (times 1 without a scale: the same value)
  m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(gs, a.nb1));
  v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(gs, gs), a.nb2));
  const float root = __fsqrt_rn(v);
  const float den = __fadd_rn(__fmul_rn(root, a.inv_sqrt_c2), a.eps);
  p = __fsub_rn(__fmul_rn(p, keep), __fmul_rn(__fdiv_rn(m, den), a.lr_c1));
  return root;
}

// Exponent of the scale of a value, biased by 127 + 8 and not yet limited: value <= 1.75 * 2^(result - 127).  A mantissa above 1.75
// carries into the exponent; infinities and NaN give 255 (the largest).
__device__ __forceinline__ uint32_t scale_exponent(const float* f) {
  const float top = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
  return min((__float_as_uint(top) + 0x1fffffu) >> 23, 255u);
}
// Codes of four elements under the group's exponent (of scale_exponent, largest of the group).  An infinite value becomes NaN, the
// one code that says "not finite".
template <bool ROOT>
__device__ __forceinline__ uint32_t encode4(const float* f, uint32_t e, uint8_t& exp_byte) {
  const int x = max(-126, min(126, (int)e - 135));
  const float inv = pow2(-x);
  float s[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) s[q] = f[q] * inv;            // exact: a power of two
  if (e >= 255u) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (fabsf(s[q]) == INFINITY) s[q] = NAN;
  }
  if (ROOT) {
    constexpr float LEAST = 0.001953125f;                   // 2^-9, the smallest code
    if (fminf(fminf(s[0], s[1]), fminf(s[2], s[3])) < LEAST) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (f[q] > 0.f) s[q] = fmaxf(s[q], LEAST);
    }
  }
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(s[0], s[1]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(s[2], s[3]), __NV_SATFINITE, __NV_E4M3);
  exp_byte = (uint8_t)(x + 127);
  return lo | hi << 16;
}
__device__ __forceinline__ void decode4(uint32_t code, uint32_t exp_byte, float* f) {
  const float scale = pow2((int)exp_byte - 127);
  const float2 lo = e4m3x2_to_f32(code), hi = e4m3x2_to_f32(code >> 16);
  f[0] = lo.x * scale; f[1] = lo.y * scale; f[2] = hi.x * scale; f[3] = hi.y * scale;
}

// What a thread reads for one step: UNITS runs of four elements, a warp's runs of one unit side by side in memory.
template <int BITS, bool P_HALF, bool G_HALF, int UNITS>
struct AdamwStep {
  Four<G_HALF> g[UNITS];
  Four<false> p[UNITS];
  Four<false> m32[BITS == 32 ? UNITS : 1], v32[BITS == 32 ? UNITS : 1];
  uint32_t mc[UNITS], vc[UNITS], mx[UNITS], vx[UNITS];      // 8 bits: codes and exponent bytes
};

// One chunk of one tensor.  FULL: all of it exists and lies on the boundaries that whole accesses need, so no step is tested.
// With 8-bit moments a thread takes two runs at a time: the exponents of their groups are then found together, two to a word.
template <int BITS, bool FULL, bool P_HALF, bool G_HALF>
__device__ __forceinline__ void adamw_chunk(const AdamwParams& a, const AdamwChunk& ch) {
  constexpr int UNITS = BITS == 8 ? 2 : 1, STEP = ADAMW_THREADS * 4 * UNITS, STEPS = ADAMW_CHUNK / STEP;
  const bool p_vec = FULL || (ch.flags & P_VEC), g_vec = FULL || (ch.flags & G_VEC);
  const float keep = (float)(1.0 - a.lr * ch.decay);
  const float scale = a.scale ? __ldg(a.scale) : 1.f;
  const int mine = (threadIdx.x >> 5) * (128 * UNITS) + (threadIdx.x & 31) * 4;      // unit u: 128 u further on
  const int left = FULL ? ADAMW_CHUNK : ch.n;
  const int padded = (left + ADAMW_GROUP - 1) / ADAMW_GROUP * ADAMW_GROUP;           // whole groups: their lanes stay together
  // this thread's first element in every array
  const int64_t flat = ch.flat + mine;
  const char* gp = reinterpret_cast<const char*>(ch.g) + mine * (G_HALF ? 2 : 4);
  char* pp = reinterpret_cast<char*>(ch.p) + mine * (P_HALF ? 2 : 4);
  float* wp = P_HALF ? a.master + flat : reinterpret_cast<float*>(pp);               // the f32 parameter
  const bool w_vec = P_HALF || p_vec;
  char* mp = reinterpret_cast<char*>(a.m) + flat * (BITS / 8);
  char* vp = reinterpret_cast<char*>(a.v) + flat * (BITS / 8);
  uint8_t *mxp = a.m_exp + flat / ADAMW_GROUP, *vxp = a.v_exp + flat / ADAMW_GROUP;
  auto count = [&](int i) { return FULL ? 4 : max(0, min(4, left - i - mine)); };    // elements of the run at i that exist
  auto held = [&](int i) { return FULL || i + mine < padded; };                      // the run lies in a group that exists

  using Step = AdamwStep<BITS, P_HALF, G_HALF, UNITS>;
  auto load = [&](int it, Step& s) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int i = it * STEP + u * 128, n = count(i);
      s.g[u] = load4<G_HALF, FULL>(gp + i * (G_HALF ? 2 : 4), g_vec, n);
      s.p[u] = load4<false, FULL>(wp + i, w_vec, n);
      if constexpr (BITS == 32) {
        const int k = held(i) ? 4 : 0;
        s.m32[u] = load4<false, FULL>(mp + i * 4, true, k);
        s.v32[u] = load4<false, FULL>(vp + i * 4, true, k);
      } else {
        const bool h = held(i);
        s.mc[u] = h ? __ldcs(reinterpret_cast<const uint32_t*>(mp + i)) : 0u;
        s.vc[u] = h ? __ldcs(reinterpret_cast<const uint32_t*>(vp + i)) : 0u;
        s.mx[u] = h ? mxp[i / ADAMW_GROUP] : 127u;
        s.vx[u] = h ? vxp[i / ADAMW_GROUP] : 127u;
      }
    }
  };
  auto work = [&](int it, const Step& s) {
    float m[UNITS][4], root[UNITS][4];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int i = it * STEP + u * 128, n = count(i);
      float g[4], p[4], v[4];
      open4<G_HALF>(s.g[u], g);
      open4<false>(s.p[u], p);
      if constexpr (BITS == 32) {
        open4<false>(s.m32[u], m[u]);
        open4<false>(s.v32[u], v);
      } else {
        decode4(s.mc[u], s.mx[u], m[u]);
        decode4(s.vc[u], s.vx[u], v);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = __fmul_rn(v[q], v[q]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) root[u][q] = adamw_element(a, scale, keep, g[q], p[q], m[u][q], v[q]);
      store4<false, FULL>(wp + i, w_vec, n, p);
      if (P_HALF) store4<true, FULL>(pp + i * 2, p_vec, n, p);
      if constexpr (BITS == 32) {
        store4<false, FULL>(mp + i * 4, true, n, m[u]);
        store4<false, FULL>(vp + i * 4, true, n, v);
      } else if (!FULL) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q >= n) m[u][q] = root[u][q] = 0.f;           // the rest of the last group holds nothing
      }
    }
    if constexpr (BITS == 8) {
      uint32_t em = scale_exponent(m[0]) | scale_exponent(m[1]) << 16, er = scale_exponent(root[0]) | scale_exponent(root[1]) << 16;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        em = __vmaxu2(em, __shfl_xor_sync(0xffffffffu, em, o));
        er = __vmaxu2(er, __shfl_xor_sync(0xffffffffu, er, o));
      }
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const int i = it * STEP + u * 128;
        uint8_t mx, rx;
        const uint32_t mc = encode4<false>(m[u], em >> 16 * u & 0xffffu, mx), rc = encode4<true>(root[u], er >> 16 * u & 0xffffu, rx);
        if (held(i)) {
          __stcs(reinterpret_cast<uint32_t*>(mp + i), mc);
          __stcs(reinterpret_cast<uint32_t*>(vp + i), rc);
          if ((threadIdx.x & 7) == 0) {
            mxp[i / ADAMW_GROUP] = mx;
            vxp[i / ADAMW_GROUP] = rx;
          }
        }
      }
    }
  };
#pragma unroll
  for (int it = 0; it < STEPS; ++it) {
    if (!FULL && it * STEP >= left) break;                  // the whole block is past the end
    Step s;
    load(it, s);
    work(it, s);
  }
}

template <int BITS, bool P_HALF, bool G_HALF>
__device__ __forceinline__ void adamw_by_edge(const AdamwParams& a, const AdamwChunk& ch) {
  if (ch.n == ADAMW_CHUNK && (ch.flags & P_VEC) && (ch.flags & G_VEC)) adamw_chunk<BITS, true, P_HALF, G_HALF>(a, ch);
  else adamw_chunk<BITS, false, P_HALF, G_HALF>(a, ch);
}

template <int BITS>
__global__ void __launch_bounds__(ADAMW_THREADS, 5) adamw_kernel(const AdamwParams a) {
  const AdamwChunk ch = a.chunks[blockIdx.x];
  if (ch.flags & P_BF16) {
    if (ch.flags & G_BF16) adamw_by_edge<BITS, true, true>(a, ch);
    else adamw_by_edge<BITS, true, false>(a, ch);
  } else {
    if (ch.flags & G_BF16) adamw_by_edge<BITS, false, true>(a, ch);
    else adamw_by_edge<BITS, false, false>(a, ch);
  }
}

// The values that 8-bit moments stand for: m_out = m, v_out = root^2.
__global__ void __launch_bounds__(256) adamw_moments_kernel(const uint8_t* __restrict__ m, const uint8_t* __restrict__ r,
                                                            const uint8_t* __restrict__ m_exp, const uint8_t* __restrict__ r_exp, int64_t n4,
                                                            float* __restrict__ m_out, float* __restrict__ v_out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    const uint32_t mc = __ldcs(reinterpret_cast<const uint32_t*>(m) + i), rc = __ldcs(reinterpret_cast<const uint32_t*>(r) + i);
    float f[4];
    decode4(mc, m_exp[i / 8], f);
    __stcs(reinterpret_cast<float4*>(m_out) + i, make_float4(f[0], f[1], f[2], f[3]));
    decode4(rc, r_exp[i / 8], f);
    __stcs(reinterpret_cast<float4*>(v_out) + i, make_float4(f[0] * f[0], f[1] * f[1], f[2] * f[2], f[3] * f[3]));
  }
}

namespace {

// Whether a parameter's memory is also another tensor's: another parameter (two blocks would write it), a gradient that some other
// block reads, or its own gradient shifted against it.  A gradient that starts where its parameter does is left alone: the thread
// that writes an element has read it (of the same type, which is the caller's to keep).
int adamw_check_overlap(const grouter_adamw_tensor* tensors, int32_t n) {
  struct Range {
    uintptr_t begin, end;
    bool written;
  };
  const std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[2 * (size_t)n]);
  if (!ranges) return GROUTER_ERR_CUDA;
  size_t count = 0;
  for (int32_t i = 0; i < n; ++i) {
    const grouter_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    const uintptr_t p = reinterpret_cast<uintptr_t>(t.param), g = reinterpret_cast<uintptr_t>(t.grad);
    const uintptr_t p_bytes = (uintptr_t)t.n * (t.param_dtype == GROUTER_BF16 ? 2 : 4), g_bytes = (uintptr_t)t.n * (t.grad_dtype == GROUTER_BF16 ? 2 : 4);
    if (p == g) {
      ranges[count++] = {p, p + std::max(p_bytes, g_bytes), true};
    } else {
      ranges[count++] = {p, p + p_bytes, true};
      ranges[count++] = {g, g + g_bytes, false};
    }
  }
  std::sort(ranges.get(), ranges.get() + count, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t written = 0, read = 0;         // where the ranges so far end
  for (size_t i = 0; i < count; ++i) {
    const Range& r = ranges[i];
    if (r.begin < written || (r.written && r.begin < read)) return GROUTER_ERR_INVALID_ARG;
    uintptr_t& end = r.written ? written : read;
    end = std::max(end, r.end);
  }
  return GROUTER_OK;
}

}  // namespace
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
  if (const int e = adamw_check_overlap(tensors, n_tensors)) return e;
  layout->n_tensors = n_tensors;
  layout->n_chunks = (int32_t)chunks;
  layout->state_elements = elements;
  layout->table_bytes = sizeof(AdamwChunk) * (size_t)chunks;
  layout->needs_master = needs_master;
  layout->reserved = 0;
  if (!table_host) return GROUTER_OK;
  if (!aligned_to(table_host, 8)) return GROUTER_ERR_MISALIGNED;
  AdamwChunk* c = static_cast<AdamwChunk*>(table_host);
  int64_t at = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const grouter_adamw_tensor& t = tensors[i];
    const bool pb = t.param_dtype == GROUTER_BF16, gb = t.grad_dtype == GROUTER_BF16;
    // a chunk starts a multiple of 16 bytes into its tensor: as well aligned as the tensor itself
    const int32_t flags = (pb ? P_BF16 : 0) | (gb ? G_BF16 : 0) | (aligned_to(t.param, pb ? 8 : 16) ? P_VEC : 0) | (aligned_to(t.grad, gb ? 8 : 16) ? G_VEC : 0);
    for (int64_t first = 0; first < t.n; first += ADAMW_CHUNK, ++c) {
      c->p = static_cast<char*>(t.param) + first * (pb ? 2 : 4);
      c->g = static_cast<const char*>(t.grad) + first * (gb ? 2 : 4);
      c->flat = at + first;
      c->decay = t.weight_decay;
      c->n = (int32_t)(t.n - first < ADAMW_CHUNK ? t.n - first : ADAMW_CHUNK);
      c->flags = flags;
    }
    at += (t.n + ADAMW_GROUP - 1) / ADAMW_GROUP * ADAMW_GROUP;
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
  a.chunks = static_cast<const AdamwChunk*>(table);
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
