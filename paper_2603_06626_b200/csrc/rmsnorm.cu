// Root-mean-square norm on a residual stream, forward and backward.
//
//   forward    h_tj = x_tj + r_tj, rounded to x's type (the stream as it goes on)      rstd_t = ((1/d) sum_j h_tj^2 + eps)^(-1/2)
//              y_tj = h_tj rstd_t w_j, in x's type or as e4m3 codes with a power-of-two scale for 128 columns (fp8.cuh)
//   backward   u = h rstd,  g = dy w
//              dx_tj = dh_tj + rstd_t (g_tj - u_tj (1/d) sum_i g_ti u_ti)      dw_j = sum_t dy_tj u_tj      (dx is also r's gradient)
//
// Every element is touched once, HBM is the bound: with bf16 the forward pass moves 8 bytes an element with the residual (7 with
// codes), the backward pass 8 with the stream's own gradient dh.  As in the layer norm a row lies in the registers of as many lanes
// as hold it in a few accesses each, and arithmetic goes two elements to an instruction.  Sums and statistics are fp32.
// Measured, bf16 with the residual: forward 32768 x 4096 159 us (6.7 TB/s), to codes 145 (6.5); 16384 x 2048 42 and 38; backward with dh 16384 x
// 2048 44 us (6.1 TB/s), f32 8192 x 16384 380 (5.7).
//   Forward: the only sum is over the rounded h, so a row takes one meeting of its threads.  Codes: the 16 (f32: 32) lanes that hold 128
//     columns find their largest value among themselves.
//   Backward: the running dw of a column stays with one thread; blocks are resident and walk over the rows, the coming ones on their
//     way into shared memory; the blocks' partial rows are added up in a fixed order (bit-reproducible, no atomics).
#include <algorithm>

#include "fp8.cuh"
#include "norm.cuh"

namespace grouter {

constexpr int RMS_MAX_D = 16384;

struct RmsForward {
  const void *x, *r, *w;
  int64_t ldx, ldr;
  int w_f32, rows, d;
  float eps;
  void *h, *y;                 // h: with a residual; y: of x's type, or codes
  uint8_t* scales;
  float* rstd;
};

// ---- forward: LANES threads a row, NP accesses of VE elements each ----
__host__ __device__ constexpr int rms_forward_threads(int lanes) { return lanes <= 32 ? 128 : lanes; }

template <typename T, int VE, int NP, int LANES, bool FP8>
__global__ void __launch_bounds__(rms_forward_threads(LANES)) rms_forward_kernel(const RmsForward p) {
  constexpr int RPB = rms_forward_threads(LANES) / LANES;
  __shared__ float red[2 * 32];
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LANES;
  const int at = threadIdx.x & (LANES - 1), d = p.d;
  after_previous_kernel();
  let_next_kernel_start();
  if (LANES >= 32 && row >= p.rows) return;      // whole warps, and whole blocks where a row has several
  const int end = LANES >= 32 || row < p.rows ? d : 0;
  const T* xr = static_cast<const T*>(p.x) + row * p.ldx;
  Pack<T, VE> q[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int c = (n * LANES + at) * VE;
    if (c < end) q[n] = ld_pack<T, VE>(xr + c);
  }
  if (p.r != nullptr) {
    const T* rr = static_cast<const T*>(p.r) + row * p.ldr;
    T* hr = static_cast<T*>(p.h) + row * d;
    Pack<T, VE> a[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int c = (n * LANES + at) * VE;
      if (c < end) a[n] = ld_pack<T, VE>(rr + c);
    }
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int c = (n * LANES + at) * VE;
      if (c < end) {
        float o[VE];
        if constexpr (VE > 1) {
#pragma unroll
          for (int i = 0; i < VE; i += 2) {
            const float2 v = add2(pair_at(q, (n * VE + i) / 2), pair_at(a, (n * VE + i) / 2));
            o[i] = v.x;
            o[i + 1] = v.y;
          }
        } else {
          o[0] = to_f32(q[n].v[0]) + to_f32(a[n].v[0]);
        }
        q[n] = make_pack<T, VE>(o);
        *reinterpret_cast<Pack<T, VE>*>(hr + c) = q[n];
      }
    }
  }
  float s[1] = {0.f};
  if constexpr (VE > 1) {
    float2 s2 = both(0.f);
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if ((n * LANES + at) * VE < end) {
#pragma unroll
        for (int i = 0; i < VE; i += 2) {
          const float2 v = pair_at(q, (n * VE + i) / 2);
          s2 = fma2(v, v, s2);
        }
      }
    s[0] = s2.x + s2.y;
  } else {
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if (n * LANES + at < end) {
        const float v = to_f32(q[n].v[0]);
        s[0] += v * v;
      }
  }
  int half = 0;
  row_sums<LANES, 1>(s, red, half);
  const float rstd = 1.f / sqrtf(s[0] * (1.f / (float)d) + p.eps);
  const int64_t across = FP8 ? fp8_atoms_across(d) : 0;
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int c = (n * LANES + at) * VE;
    float o[VE];
    if (c < end) {
      float wl[VE];
      if (p.w_f32) load_weights<float, VE>(static_cast<const float*>(p.w), c, wl);
      else load_weights<__nv_bfloat16, VE>(static_cast<const __nv_bfloat16*>(p.w), c, wl);
      if constexpr (VE > 1) {
#pragma unroll
        for (int i = 0; i < VE; i += 2) {
          const float2 v = mul2(mul2(pair_at(q, (n * VE + i) / 2), both(rstd)), make_float2(wl[i], wl[i + 1]));
          o[i] = v.x;
          o[i + 1] = v.y;
        }
      } else {
        o[0] = to_f32(q[n].v[0]) * rstd * wl[0];
      }
      if constexpr (!FP8) st_pack<T, VE>(static_cast<T*>(p.y) + row * d + c, o);
    }
    if constexpr (FP8) {
      constexpr int GROUP = FP8_BLOCK / VE;      // lanes that share a scale
      static_assert(LANES >= GROUP && GROUP <= 32, "a block of columns lies in one warp");
      float top = 0.f;
      if (c < end) {
#pragma unroll
        for (int i = 0; i < VE; ++i) top = larger(top, o[i]);
      }
      top = lanes_top<GROUP>(top);
      const bool inf = __any_sync(0xffffffffu, not_finite(top));
      if (inf) {
        top = 0.f;
        if (c < end) {
#pragma unroll
          for (int i = 0; i < VE; ++i) top = larger_finite(top, o[i]);
        }
        top = lanes_top<GROUP>(top);
      }
      const uint32_t e = fp8_exponent(top);
      const float inv = fp8_inverse(e);
      if (c < end) {
        uint8_t* to = static_cast<uint8_t*>(p.y) + row * d + c;
        uint32_t q[VE / 4];
#pragma unroll
        for (int i = 0; i < VE; i += 4) q[i / 4] = inf ? fp8_quad<true>(o + i, inv) : fp8_quad<false>(o + i, inv);
        if constexpr (VE == 8) *reinterpret_cast<uint2*>(to) = make_uint2(q[0], q[1]);
        else *reinterpret_cast<uint32_t*>(to) = q[0];
        if (at % GROUP == 0) p.scales[fp8_scale_at(row, c / FP8_BLOCK, across)] = (uint8_t)e;
      }
    }
  }
  if (at == 0 && row < p.rows && p.rstd) p.rstd[row] = rstd;
}

// ---- backward: TPR threads a row, RMS_EPT elements each ----
constexpr int RMS_EPT = 16;
__host__ __device__ constexpr int rms_backward_threads(int tpr) { return tpr <= 32 ? 256 : tpr; }
__host__ __device__ constexpr int rms_backward_per_sm(int tpr) { return tpr >= 512 ? 1 : 512 / rms_backward_threads(tpr); }
// Rows (h, dy and, with the stream's gradient, dh) that a block has on their way or in use, as many as shared memory takes.
__host__ __device__ constexpr int rms_ring(int bytes, int tpr, bool dh) {
  return tpr == 1024 ? (bytes == 2 ? (dh ? 2 : 3) : 1) : bytes == 2 ? 4 : (dh ? 2 : 3);
}

struct RmsBackward {
  const void *dy, *h, *dh, *w;
  int64_t ldh;
  int w_f32, rows, d;
  const float* rstd;
  void* dx;
  float* partial;
};

// Every thread copies its own elements of the coming rows into shared memory and reads back only those: the ring needs no barrier.
// Rows that are not 16-byte aligned: plain loads, no ring.
template <typename T, typename W, int VE, int TPR, bool DH>
__global__ void __launch_bounds__(rms_backward_threads(TPR), rms_backward_per_sm(TPR)) rms_backward_kernel(const RmsBackward p) {
  constexpr int NV = RMS_EPT / VE, PAIRS = RMS_EPT / 2, NS = DH ? 3 : 2;
  constexpr int THREADS = rms_backward_threads(TPR), RPB = THREADS / TPR;
  constexpr bool RING = VE * sizeof(T) == 16;
  constexpr int S = rms_ring(sizeof(T), TPR, DH);
  constexpr bool HOLD = TPR < 1024;     // the weights stay in registers (1024 threads have 64 each: there they are read from L1)
  extern __shared__ uint4 s_ring[];     // RING: [S][h, dy, dh][NV][THREADS]; at the end the columns of the block's rows
  __shared__ float red[2 * 32];
  const int lane = threadIdx.x & (TPR - 1), sub = threadIdx.x / TPR, d = p.d;
  const float inv_d = 1.f / (float)d;
  const T* base[3] = {static_cast<const T*>(p.h), static_cast<const T*>(p.dy), static_cast<const T*>(p.dh)};
  const int64_t ld[3] = {p.ldh, d, d};
  after_previous_kernel();
  // pair j holds elements 2j and 2j + 1 of a thread's [NV][VE]; columns beyond d hold zeros throughout
  auto weights = [&](float2 (&f)[PAIRS]) {
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      float t[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) t[i] = 0.f;
      const int c = (n * TPR + lane) * VE;
      if (c < d) load_weights<W, VE>(static_cast<const W*>(p.w), c, t);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const int k = n * VE + i;
        if (k & 1) f[k / 2].y = t[i];
        else f[k / 2].x = t[i];
      }
    }
  };
  float2 wv[PAIRS], aw[PAIRS];
  if constexpr (HOLD) weights(wv);
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) aw[j] = both(0.f);

  auto slot = [&](int s, int which, int n) { return s_ring + ((s * NS + which) * NV + n) * THREADS + threadIdx.x; };
  auto fetch = [&](int64_t r, int s) {
    if (r < p.rows) {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const int c = (n * TPR + lane) * VE;
        if (c < d) {
#pragma unroll
          for (int k = 0; k < NS; ++k) copy16_async(slot(s, k, n), base[k] + r * ld[k] + c);
        }
      }
    }
    copies_commit();
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  const int64_t step = (int64_t)gridDim.x * RPB;
  float next_rstd = row < p.rows ? __ldg(p.rstd + row) : 0.f;
  if constexpr (RING) {
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if ((n * TPR + lane) * VE >= d)
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int k = 0; k < NS; ++k) *slot(s, k, n) = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(row + s * step, s);
  }
  int half = 0, s_at = 0;
  // rows that share a warp stay together for their sums: those past the last row hold zeros
  const int behind = TPR < 32 ? sub & (32 / TPR - 1) : 0;
  for (; row - behind < p.rows; row += step) {
    const bool live = TPR >= 32 || row < p.rows;
    const float rstd = live ? next_rstd : 0.f;
    if (row + step < p.rows) next_rstd = __ldg(p.rstd + row + step);
    auto take = [&](Pack<T, VE> (&v)[NV], int which) {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        if constexpr (RING) {
          *reinterpret_cast<uint4*>(&v[n]) = live ? *slot(s_at, which, n) : make_uint4(0u, 0u, 0u, 0u);
        } else {
          const int c = (n * TPR + lane) * VE;
#pragma unroll
          for (int i = 0; i < VE; ++i) v[n].v[i] = from_f32<T>(0.f);
          if (c < d && live) v[n] = ld_pack<T, VE>(base[which] + row * ld[which] + c);
        }
      }
    };
    Pack<T, VE> ph[NV], pg[NV], pd[NV];
    if constexpr (RING) copies_wait<S - 1>();
    take(ph, 0);
    take(pg, 1);
    if constexpr (DH && !RING) take(pd, 2);      // on its way while the sum is taken
    if constexpr (!HOLD) weights(wv);
    float2 s2 = both(0.f);
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      const float2 g = pair_at(pg, j), h = pair_at(ph, j);
      aw[j] = fma2(g, mul2(h, both(rstd)), aw[j]);
      s2 = fma2(mul2(g, wv[j]), h, s2);
    }
    float s[1] = {s2.x + s2.y};
    row_sums<TPR, 1>(s, red, half);
    // dx = dh + rstd g - h rstd^3 mean(g h)
    const float2 r1 = both(rstd), c2 = both(-s[0] * inv_d * rstd * rstd * rstd);
    if constexpr (!HOLD) {
      asm volatile("" ::: "memory");
      weights(wv);
      if constexpr (RING) {
        take(ph, 0);
        take(pg, 1);
      }
    }
    if constexpr (DH && RING) take(pd, 2);
    T* dr = static_cast<T*>(p.dx) + row * d;
    float o[RMS_EPT];
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      float2 v = mul2(pair_at(ph, j), c2);
      v = fma2(mul2(pair_at(pg, j), wv[j]), r1, v);
      if constexpr (DH) v = add2(v, pair_at(pd, j));
      o[2 * j] = v.x;
      o[2 * j + 1] = v.y;
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d && live) st_pack<T, VE>(dr + c, o + n * VE);
    }
    if constexpr (RING) {
      fetch(row + S * step, s_at);
      s_at = s_at + 1 == S ? 0 : s_at + 1;
    }
  }
  let_next_kernel_start();
  float* out = p.partial + (int64_t)blockIdx.x * d;
  auto put_columns = [&](float* to) {
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) store_floats<VE>(to + c, [&](int i) { return (n * VE + i) & 1 ? aw[(n * VE + i) / 2].y : aw[(n * VE + i) / 2].x; });
    }
  };
  if constexpr (RPB == 1) {
    put_columns(out);
  } else {
    // the columns of each of the rows that the block works on at a time take the ring's place (nothing is on its way into it)
    float* cols = reinterpret_cast<float*>(s_ring);
    __syncthreads();
    put_columns(cols + sub * d);
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += THREADS) {
      float a = cols[c];
#pragma unroll
      for (int r = 1; r < RPB; ++r) a += cols[r * d + c];
      out[c] = a;
    }
  }
}

namespace {

// Threads that hold a row of d elements in the backward pass.
int rms_tpr(int d) {
  int tpr = 8;
  while (tpr * RMS_EPT < d) tpr *= 2;
  return tpr;
}
// Blocks of the backward pass: each leaves a partial row, which has to be written and read again, so a block works on RMS_WALK rows before
// every SM gets another one (1000 x 1024 bf16: 7.0 us, a row a block 9.4; 1001 x 1023 f32 8.9 and 10.0), and all SMs have equally many
// (2000 x 2048 with 592 blocks 8.3 us, with 500 11.1).
constexpr int RMS_WALK = 4;
int rms_backward_blocks(int rows, int d) {
  const int tpr = rms_tpr(d), rpb = rms_backward_threads(tpr) / tpr;
  const int want = (rows + rpb - 1) / rpb, cap = current_sms() * rms_backward_per_sm(tpr);
  const int sms = std::max(1, current_sms()), a_sm = (want + RMS_WALK * sms - 1) / (RMS_WALK * sms);
  return std::max(1, std::min({want, cap, a_sm * sms}));
}

template <typename T, int VE, int NP, int LANES, bool FP8>
cudaError_t forward_launch(const RmsForward& a, cudaStream_t st) {
  constexpr int THREADS = rms_forward_threads(LANES), RPB = THREADS / LANES;
  return launch_dependent(rms_forward_kernel<T, VE, NP, LANES, FP8>, dim3((a.rows + RPB - 1) / RPB), dim3(THREADS), 0, st, a);
}

// Up to FEW accesses a lane while a quarter of a warp holds a row (codes: as many lanes as share a scale), then more lanes; a warp's
// lanes then take up to MOST, more warps follow up to LAST lanes, those take twice MOST, and what is still needed of both.
template <typename T, int VE, bool FP8, int MOST, int FEW, int LAST, int NP = 1, int LANES = FP8 ? FP8_BLOCK / VE : 8>
cudaError_t forward_spread(const RmsForward& a, cudaStream_t st) {
  constexpr int HOLDS = NP * LANES * VE;
  if constexpr (HOLDS < RMS_MAX_D) {
    if (a.d > HOLDS) {
      constexpr bool more = NP < FEW || (LANES >= 32 && (NP < MOST || (LANES == LAST && NP < 2 * MOST) || (LANES == 512 && NP < 16)));
      if constexpr (more) return forward_spread<T, VE, FP8, MOST, FEW, LAST, 2 * NP, LANES>(a, st);
      else return forward_spread<T, VE, FP8, MOST, FEW, LAST, NP, 2 * LANES>(a, st);
    }
  }
  return forward_launch<T, VE, NP, LANES, FP8>(a, st);
}

template <typename T, int VE, bool FP8>
cudaError_t forward_by_width(const RmsForward& a, cudaStream_t st) {
  if constexpr (VE * sizeof(T) < 16) {
    return forward_spread<T, VE, FP8, 8, 4, 512>(a, st);
  } else {
    // two accesses a lane as long as a block of 256 holds the row: more warps with less each are ahead of four (16384 x 2048 to codes 38.1 and
    // 40.1 us, to bf16 41.9 and 42.8; 4096 x 16384 to codes 77.7 and 86.6) and of one (42.2, 42.3)
    return (int64_t)a.rows * a.d <= (1 << 21) ? forward_spread<T, VE, FP8, 2, 1, 512>(a, st) : forward_spread<T, VE, FP8, 2, 2, 256>(a, st);
  }
}

template <typename T>
cudaError_t forward_by_type(const RmsForward& a, bool fp8, cudaStream_t st) {
  // accesses of VE elements where every row of every activation and the weights start on a boundary of them
  auto fits = [&](int ve) {
    const size_t b = ve * sizeof(T), wb = std::min<size_t>(ve * (a.w_f32 ? 4 : 2), 16);
    return a.d % ve == 0 && a.ldx % ve == 0 && a.ldr % ve == 0 && aligned_to(a.x, b) && aligned_to(a.r, b) && aligned_to(a.h, b) &&
           (fp8 || aligned_to(a.y, b)) && aligned_to(a.w, wb);
  };
  if (fp8) return fits(vec16<T>()) ? forward_by_width<T, vec16<T>(), true>(a, st) : cudaErrorInvalidValue;
  if (fits(vec16<T>())) return forward_by_width<T, vec16<T>(), false>(a, st);
  if (fits(2)) return forward_by_width<T, 2, false>(a, st);
  return forward_by_width<T, 1, false>(a, st);
}

template <typename T, typename W, int VE, int TPR, bool DH>
cudaError_t backward_launch(const RmsBackward& a, int blocks, cudaStream_t st) {
  constexpr int threads = rms_backward_threads(TPR);
  constexpr int ring = VE == vec16<T>() ? rms_ring(sizeof(T), TPR, DH) * (DH ? 3 : 2) * (RMS_EPT / VE) * threads * 16 : 0;
  constexpr int cols = threads * RMS_EPT * (int)sizeof(float);
  constexpr int smem = ring > cols ? ring : cols;      // up to 192 KB
  auto kern = rms_backward_kernel<T, W, VE, TPR, DH>;
  static bool configured[64] = {};                     // the opt-in is a per-device setting
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  return launch_dependent(kern, dim3(blocks), dim3(threads), smem, st, a);
}

template <typename T, typename W, int VE, bool DH>
cudaError_t backward_by_width(const RmsBackward& a, int blocks, cudaStream_t st) {
  switch (rms_tpr(a.d)) {
    case 8: return backward_launch<T, W, VE, 8, DH>(a, blocks, st);
    case 16: return backward_launch<T, W, VE, 16, DH>(a, blocks, st);
    case 32: return backward_launch<T, W, VE, 32, DH>(a, blocks, st);
    case 64: return backward_launch<T, W, VE, 64, DH>(a, blocks, st);
    case 128: return backward_launch<T, W, VE, 128, DH>(a, blocks, st);
    case 256: return backward_launch<T, W, VE, 256, DH>(a, blocks, st);
    case 512: return backward_launch<T, W, VE, 512, DH>(a, blocks, st);
    default: return backward_launch<T, W, VE, 1024, DH>(a, blocks, st);
  }
}
template <typename T, typename W, int VE>
cudaError_t backward_by_stream(const RmsBackward& a, int blocks, cudaStream_t st) {
  return a.dh ? backward_by_width<T, W, VE, true>(a, blocks, st) : backward_by_width<T, W, VE, false>(a, blocks, st);
}
template <typename T, int VE>
cudaError_t backward_by_weights(const RmsBackward& a, int blocks, cudaStream_t st) {
  return a.w_f32 ? backward_by_stream<T, float, VE>(a, blocks, st) : backward_by_stream<T, __nv_bfloat16, VE>(a, blocks, st);
}
template <typename T>
cudaError_t backward_by_type(const RmsBackward& a, int blocks, cudaStream_t st) {
  auto fits = [&](int ve) {
    const size_t b = ve * sizeof(T), wb = std::min<size_t>(ve * (a.w_f32 ? 4 : 2), 16);
    return a.d % ve == 0 && a.ldh % ve == 0 && aligned_to(a.h, b) && aligned_to(a.dy, b) && aligned_to(a.dh, b) && aligned_to(a.dx, b) &&
           aligned_to(a.w, wb);
  };
  if (fits(vec16<T>())) return backward_by_weights<T, vec16<T>()>(a, blocks, st);
  if (fits(2)) return backward_by_weights<T, 2>(a, blocks, st);
  return backward_by_weights<T, 1>(a, blocks, st);
}

int rms_check(int32_t rows, int32_t d, int64_t ldx, int32_t dtype, int32_t w_dtype) {
  if (rows < 0 || d < 1 || ldx < d) return GROUTER_ERR_INVALID_ARG;
  if ((dtype != GROUTER_BF16 && dtype != GROUTER_F32) || (w_dtype != GROUTER_BF16 && w_dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  return d > RMS_MAX_D || rows > INT32_MAX - (1 << 20) ? GROUTER_ERR_UNSUPPORTED : GROUTER_OK;
}

}  // namespace
}  // namespace grouter

using namespace grouter;

extern "C" {

int grouter_rmsnorm_fwd(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* w, int32_t rows, int32_t d, int32_t dtype,
                        int32_t w_dtype, float eps, void* h, void* y, void* scales, float* rstd, void* stream) {
  if (!w || !(eps >= 0.f) || (rows > 0 && (!x || !y || (residual && !h)))) return GROUTER_ERR_INVALID_ARG;
  if (const int e = rms_check(rows, d, ldx, dtype, w_dtype)) return e;
  if (residual && ldr < d) return GROUTER_ERR_INVALID_ARG;
  const size_t el = dtype == GROUTER_F32 ? 4 : 2, wl = w_dtype == GROUTER_F32 ? 4 : 2;
  if (!aligned_to(x, el) || !aligned_to(residual, el) || !aligned_to(h, el) || !aligned_to(w, wl) || !aligned_to(rstd, 4)) return GROUTER_ERR_MISALIGNED;
  if (scales) {
    if (d % 16) return GROUTER_ERR_UNSUPPORTED;
    if (!aligned_to(x, 16) || !aligned_to(residual, 16) || !aligned_to(h, 16) || !aligned_to(y, 16) || !aligned_to(w, 16) || !aligned_to(scales, 16) ||
        ldx * el % 16 || (residual && ldr * el % 16))
      return GROUTER_ERR_MISALIGNED;
  } else if (!aligned_to(y, el)) {
    return GROUTER_ERR_MISALIGNED;
  }
  if (rows == 0) return GROUTER_OK;
  RmsForward a{};
  a.x = x; a.ldx = ldx; a.r = residual; a.ldr = residual ? ldr : 0; a.w = w; a.w_f32 = w_dtype == GROUTER_F32; a.rows = rows; a.d = d; a.eps = eps;
  a.h = residual ? h : nullptr; a.y = y; a.scales = static_cast<uint8_t*>(scales); a.rstd = rstd;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == GROUTER_F32 ? forward_by_type<float>(a, scales != nullptr, st) : forward_by_type<__nv_bfloat16>(a, scales != nullptr, st);
  return e == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

size_t grouter_rmsnorm_bwd_workspace_bytes(int32_t rows, int32_t d) {
  if (rms_check(rows, d, d, GROUTER_BF16, GROUTER_BF16) != GROUTER_OK) return 0;
  return (size_t)rms_backward_blocks(rows, d) * d * sizeof(float);
}

int grouter_rmsnorm_bwd(const void* dy, const void* h, int64_t ldh, const void* dh, const void* w, const float* rstd, int32_t rows, int32_t d,
                        int32_t dtype, int32_t w_dtype, void* dx, float* dw, void* workspace, void* stream) {
  if (!w || !dw || (rows > 0 && (!dy || !h || !rstd || !dx || !workspace))) return GROUTER_ERR_INVALID_ARG;
  if (const int e = rms_check(rows, d, ldh, dtype, w_dtype)) return e;
  const size_t el = dtype == GROUTER_F32 ? 4 : 2, wl = w_dtype == GROUTER_F32 ? 4 : 2;
  if (!aligned_to(h, el) || !aligned_to(dy, el) || !aligned_to(dh, el) || !aligned_to(dx, el) || !aligned_to(w, wl) || !aligned_to(rstd, 4) ||
      !aligned_to(dw, 4) || !aligned_to(workspace, 16))
    return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) return cudaMemsetAsync(dw, 0, (size_t)d * 4, st) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
  RmsBackward a{};
  a.dy = dy; a.h = h; a.ldh = ldh; a.dh = dh; a.w = w; a.w_f32 = w_dtype == GROUTER_F32; a.rows = rows; a.d = d; a.rstd = rstd;
  a.dx = dx; a.partial = static_cast<float*>(workspace);
  const int blocks = rms_backward_blocks(rows, d);
  const cudaError_t e = dtype == GROUTER_F32 ? backward_by_type<float>(a, blocks, st) : backward_by_type<__nv_bfloat16>(a, blocks, st);
  if (e != cudaSuccess) return GROUTER_ERR_CUDA;
  return launch_sum_rows(a.partial, blocks, d, dw, d, nullptr, st) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
