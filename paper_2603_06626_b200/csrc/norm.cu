// Layer norm over the rows of a matrix, forward and backward.
//
//   forward    mean_t = (1/d) sum_j x_tj     rstd_t = ((1/d) sum_j (x_tj - mean_t)^2 + eps)^(-1/2)
//              y_tj = (x_tj - mean_t) rstd_t w_j + b_j
//   backward   h = (x - mean) rstd,  g = dy w
//              dx_tj = rstd_t (g_tj - (1/d) sum_i g_ti - h_tj (1/d) sum_i g_ti h_ti)
//              dw_j = sum_t dy_tj h_tj       db_j = sum_t dy_tj
//
// Both passes touch every element once and are bound by HBM.  A row is held in registers, NORM_EPT elements a thread, by a
// warp (narrow rows) or a whole block; sums are taken in fp32 from the registers, the variance from the centred values
// (never as a difference of large sums).  Blocks are resident and walk over the rows, so a thread always sees the same
// columns: the weights are read once per block, and the backward pass adds up dw and db of its columns in registers and
// writes one partial row per block, which a second small kernel adds up in a fixed order (bit-reproducible, no atomics).
#include "vec.cuh"

namespace grouter {

constexpr int NORM_EPT = 16;            // elements of a row that a thread holds
constexpr int NORM_MAX_D = 1024 * NORM_EPT;
constexpr int NORM_WARP_ROWS = 8;       // rows of a block that gives every row one warp

template <int TPR>
constexpr int norm_threads() { return TPR == 32 ? 32 * NORM_WARP_ROWS : TPR; }

// Sum over the TPR threads of a row, the same value in each of them.  `red` has two halves used in turn: a warp may still
// read one while the others already write the next sum into the other, and the barrier in between keeps the third away.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& half) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lanes_sum<32>(v[n]);
  if constexpr (TPR > 32) {
    constexpr int NW = TPR / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* buf = red + half * (2 * 32);
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

// VE consecutive weights from column c on (zeros without weights or beyond d), of either type; in whole 16- or 8-byte
// accesses where VE > 1, which the host only picks when the weights start on a 16-byte boundary.
template <int VE>
__device__ __forceinline__ void load_weights(const void* w, int w_f32, int c, int d, float (&f)[VE]) {
#pragma unroll
  for (int i = 0; i < VE; ++i) f[i] = 0.f;
  if (w == nullptr || c >= d) return;
  if (w_f32) {
    const float* p = reinterpret_cast<const float*>(w) + c;
    if constexpr (VE == 1) {
      f[0] = __ldg(p);
    } else {
#pragma unroll
      for (int q = 0; q < VE; q += 4) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(p + q));
        f[q] = v.x;
        f[q + 1] = v.y;
        f[q + 2] = v.z;
        f[q + 3] = v.w;
      }
    }
  } else {
    const __nv_bfloat16* p = reinterpret_cast<const __nv_bfloat16*>(w) + c;
    if constexpr (VE == 1) {
      f[0] = __bfloat162float(*p);
    } else {
#pragma unroll
      for (int q = 0; q < VE; q += 4) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(p + q));
        const float2 lo = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.x));
        const float2 hi = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.y));
        f[q] = lo.x;
        f[q + 1] = lo.y;
        f[q + 2] = hi.x;
        f[q + 3] = hi.y;
      }
    }
  }
}

template <typename T, int VE, int TPR>
__global__ void __launch_bounds__(norm_threads<TPR>()) norm_forward_kernel(const T* __restrict__ x, int64_t ldx, const void* __restrict__ w,
                                                                           const void* __restrict__ b, int w_f32, int rows, int d, float eps,
                                                                           T* __restrict__ y, float* __restrict__ mean_out,
                                                                           float* __restrict__ rstd_out) {
  constexpr int NV = NORM_EPT / VE;
  constexpr int RPB = TPR == 32 ? NORM_WARP_ROWS : 1;
  __shared__ float red[2 * 2 * 32];
  const int lane = threadIdx.x & (TPR - 1);
  const int sub = TPR == 32 ? threadIdx.x >> 5 : 0;
  const float inv_d = 1.f / (float)d;
  float wv[NV][VE], bv[NV][VE];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = (n * TPR + lane) * VE;
    load_weights<VE>(w, w_f32, c, d, wv[n]);
    load_weights<VE>(b, w_f32, c, d, bv[n]);
  }
  int half = 0;
  for (int row = blockIdx.x * RPB + sub; row < rows; row += gridDim.x * RPB) {
    const T* xr = x + (int64_t)row * ldx;
    float v[NV][VE];
    float s[1] = {0.f};
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) {
        const Pack<T, VE> p = ld_pack<T, VE>(xr + c);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          v[n][i] = to_f32(p.v[i]);
          s[0] += v[n][i];
        }
      }
    }
    row_sums<TPR, 1>(s, red, half);
    const float mean = s[0] * inv_d;
    float q[1] = {0.f};
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if ((n * TPR + lane) * VE < d) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          v[n][i] -= mean;
          q[0] += v[n][i] * v[n][i];
        }
      }
    }
    row_sums<TPR, 1>(q, red, half);
    const float rstd = 1.f / sqrtf(q[0] * inv_d + eps);
    T* yr = y + (int64_t)row * d;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) {
        float o[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) o[i] = v[n][i] * rstd * wv[n][i] + bv[n][i];
        st_pack<T, VE>(yr + c, o);
      }
    }
    if (lane == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
  }
}

// WIDE (1024 threads a row, 64 registers each): the running dw and db live in shared memory instead of registers, each
// thread touching only its own columns, and the weights are read again for every row (they stay in L1 / L2).
template <typename T, int VE, int TPR>
__global__ void __launch_bounds__(norm_threads<TPR>()) norm_backward_kernel(const T* __restrict__ dy, const T* __restrict__ x, int64_t ldx,
                                                                            const void* __restrict__ w, int w_f32, const float* __restrict__ mean_in,
                                                                            const float* __restrict__ rstd_in, int rows, int d, T* __restrict__ dx,
                                                                            float* __restrict__ partial) {
  constexpr int NV = NORM_EPT / VE;
  constexpr int RPB = TPR == 32 ? NORM_WARP_ROWS : 1;
  constexpr bool WIDE = TPR == 1024;
  extern __shared__ float s_cols[];     // WIDE: [2][NORM_EPT][TPR], a column of it for each thread;  one warp per row: [NORM_WARP_ROWS][32 * NORM_EPT]
  __shared__ float red[2 * 2 * 32];
  const int lane = threadIdx.x & (TPR - 1);
  const int sub = TPR == 32 ? threadIdx.x >> 5 : 0;
  const float inv_d = 1.f / (float)d;
  float wv[WIDE ? 1 : NV][VE], aw[WIDE ? 1 : NV][VE], ab[WIDE ? 1 : NV][VE];
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < 2 * NORM_EPT; ++i) s_cols[i * TPR + lane] = 0.f;
  } else {
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      load_weights<VE>(w, w_f32, (n * TPR + lane) * VE, d, wv[n]);
#pragma unroll
      for (int i = 0; i < VE; ++i) aw[n][i] = ab[n][i] = 0.f;
    }
  }
  int half = 0;
  for (int row = blockIdx.x * RPB + sub; row < rows; row += gridDim.x * RPB) {
    const T* xr = x + (int64_t)row * ldx;
    const T* gr = dy + (int64_t)row * d;
    const float mean = __ldg(mean_in + row), rstd = __ldg(rstd_in + row);
    Pack<T, VE> px[NV], pg[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) {
        px[n] = ld_pack<T, VE>(xr + c);
        pg[n] = ld_pack<T, VE>(gr + c);
      }
    }
    float s[2] = {0.f, 0.f};            // sum of g, sum of g h
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) {
        float wl[VE];
        if constexpr (WIDE) load_weights<VE>(w, w_f32, c, d, wl);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const float g0 = to_f32(pg[n].v[i]), h = (to_f32(px[n].v[i]) - mean) * rstd;
          if constexpr (WIDE) {
            s_cols[(n * VE + i) * TPR + lane] += g0 * h;
            s_cols[(NORM_EPT + n * VE + i) * TPR + lane] += g0;
          } else {
            aw[n][i] += g0 * h;
            ab[n][i] += g0;
            wl[i] = wv[n][i];
          }
          s[0] += g0 * wl[i];
          s[1] += g0 * wl[i] * h;
        }
      }
    }
    row_sums<TPR, 2>(s, red, half);
    const float c1 = s[0] * inv_d, c2 = s[1] * inv_d;
    T* dr = dx + (int64_t)row * d;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) {
        float wl[VE], o[VE];
        if constexpr (WIDE) load_weights<VE>(w, w_f32, c, d, wl);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          if constexpr (!WIDE) wl[i] = wv[n][i];
          const float h = (to_f32(px[n].v[i]) - mean) * rstd;
          o[i] = rstd * (to_f32(pg[n].v[i]) * wl[i] - c1 - h * c2);
        }
        st_pack<T, VE>(dr + c, o);
      }
    }
  }
  let_next_kernel_start();
  // this block's partial row: [dw | db]
  float* pw = partial + (int64_t)blockIdx.x * 2 * d;
  if constexpr (WIDE) {
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const int c = (n * TPR + lane) * VE + i;
        if (c < d) {
          pw[c] = s_cols[(n * VE + i) * TPR + lane];
          pw[d + c] = s_cols[(NORM_EPT + n * VE + i) * TPR + lane];
        }
      }
  } else if constexpr (TPR == 32) {
    constexpr int COLS = 32 * NORM_EPT;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int i = 0; i < VE; ++i) s_cols[sub * COLS + (n * 32 + lane) * VE + i] = pass == 0 ? aw[n][i] : ab[n][i];
      __syncthreads();
      for (int c = threadIdx.x; c < d; c += 32 * NORM_WARP_ROWS) {
        float a = 0.f;
#pragma unroll
        for (int r = 0; r < NORM_WARP_ROWS; ++r) a += s_cols[r * COLS + c];
        pw[pass * d + c] = a;
      }
      __syncthreads();
    }
  } else {
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const int c = (n * TPR + lane) * VE + i;
        if (c < d) {
          pw[c] = aw[n][i];
          pw[d + c] = ab[n][i];
        }
      }
  }
}

// Column sums of `n_part` rows of `cols` values, in a fixed order: a block takes 32 columns, its 32 warps share the rows.
// The first n0 columns go to out0, the others to out1 (which may be null).
__global__ void __launch_bounds__(1024) sum_rows_kernel(const float* __restrict__ partial, int n_part, int cols, float* __restrict__ out0, int n0,
                                                        float* __restrict__ out1) {
  __shared__ float s[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float a = 0.f;
  after_previous_kernel();
  if (c < cols) {
#pragma unroll 8
    for (int r = warp; r < n_part; r += 32) a += partial[(int64_t)r * cols + c];
  }
  s[warp][lane] = a;
  __syncthreads();
  const float v = lanes_sum<32>(s[lane][warp]);
  const int oc = blockIdx.x * 32 + warp;
  if (lane == 0 && oc < cols) {
    if (oc < n0) out0[oc] = v;
    else if (out1) out1[oc - n0] = v;
  }
}

cudaError_t launch_sum_rows(const float* partial, int n_part, int cols, float* out0, int n0, float* out1, cudaStream_t st) {
  return launch_dependent(sum_rows_kernel, dim3((cols + 31) / 32), dim3(1024), 0, st, partial, n_part, cols, out0, n0, out1);
}

namespace {

struct NormArgs {
  const void *x, *dy, *w, *b;
  int64_t ldx;
  int w_f32, rows, d;
  float eps;
  const float *mean_in, *rstd_in;
  void *y, *dx;
  float *mean_out, *rstd_out, *partial, *dw, *db;
  cudaStream_t st;
};

// Threads that hold a row of d elements.
int norm_tpr(int d) {
  if (d <= 32 * NORM_EPT) return 32;
  if (d <= 128 * NORM_EPT) return 128;
  if (d <= 256 * NORM_EPT) return 256;
  if (d <= 512 * NORM_EPT) return 512;
  return 1024;
}

// Blocks of the backward pass: enough to fill the GPU at the registers the kernels take, and no more than there are
// rows, since every block leaves a partial row behind.
int norm_backward_blocks(int rows, int d) {
  const int sms = current_sms();
  const int tpr = norm_tpr(d);
  const int rpb = tpr == 32 ? NORM_WARP_ROWS : 1;
  const int per_sm = tpr <= 128 ? (tpr == 32 ? 2 : 4) : tpr == 256 ? 2 : 1;
  const int want = (rows + rpb - 1) / rpb;
  return want < sms * per_sm ? want : sms * per_sm;
}

template <typename T, int VE, int TPR>
cudaError_t forward_launch(const NormArgs& a) {
  constexpr int RPB = TPR == 32 ? NORM_WARP_ROWS : 1;
  const int per_sm = 2048 / norm_threads<TPR>();
  const int want = (a.rows + RPB - 1) / RPB, cap = current_sms() * per_sm;
  norm_forward_kernel<T, VE, TPR><<<want < cap ? want : cap, norm_threads<TPR>(), 0, a.st>>>(
      static_cast<const T*>(a.x), a.ldx, a.w, a.b, a.w_f32, a.rows, a.d, a.eps, static_cast<T*>(a.y), a.mean_out, a.rstd_out);
  return cudaGetLastError();
}

template <typename T, int VE, int TPR>
cudaError_t backward_launch(const NormArgs& a) {
  const int nblk = norm_backward_blocks(a.rows, a.d);
  const size_t smem = TPR == 1024 ? sizeof(float) * 2 * NORM_EPT * TPR : TPR == 32 ? sizeof(float) * NORM_WARP_ROWS * 32 * NORM_EPT : 0;
  auto kern = norm_backward_kernel<T, VE, TPR>;
  if (TPR == 1024) {      // up to 128 KB: the opt-in is a per-device setting
    static bool configured[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !configured[dev]) {
      const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      if (e != cudaSuccess) return e;
      if (dev >= 0 && dev < 64) configured[dev] = true;
    }
  }
  kern<<<nblk, norm_threads<TPR>(), smem, a.st>>>(static_cast<const T*>(a.dy), static_cast<const T*>(a.x), a.ldx, a.w, a.w_f32, a.mean_in,
                                                  a.rstd_in, a.rows, a.d, static_cast<T*>(a.dx), a.partial);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_sum_rows(a.partial, nblk, 2 * a.d, a.dw, a.d, a.db, a.st);
}

template <typename T, int VE, bool BACKWARD>
cudaError_t norm_by_width(const NormArgs& a) {
  switch (norm_tpr(a.d)) {
    case 32: return BACKWARD ? backward_launch<T, VE, 32>(a) : forward_launch<T, VE, 32>(a);
    case 128: return BACKWARD ? backward_launch<T, VE, 128>(a) : forward_launch<T, VE, 128>(a);
    case 256: return BACKWARD ? backward_launch<T, VE, 256>(a) : forward_launch<T, VE, 256>(a);
    case 512: return BACKWARD ? backward_launch<T, VE, 512>(a) : forward_launch<T, VE, 512>(a);
    default: return BACKWARD ? backward_launch<T, VE, 1024>(a) : forward_launch<T, VE, 1024>(a);
  }
}

// 16-byte accesses where every row of every activation and the weights start on a 16-byte boundary, single elements otherwise.
template <bool BACKWARD>
cudaError_t norm_dispatch(const NormArgs& a, int dtype) {
  const int ve = dtype == GROUTER_F32 ? vec16<float>() : vec16<__nv_bfloat16>();
  const bool vec = a.d % ve == 0 && a.ldx % ve == 0 && aligned_to(a.x, 16) && aligned_to(BACKWARD ? a.dy : a.y, 16) &&
                   (!BACKWARD || aligned_to(a.dx, 16)) && aligned_to(a.w, 16) && aligned_to(a.b, 16);
  if (dtype == GROUTER_F32) return vec ? norm_by_width<float, vec16<float>(), BACKWARD>(a) : norm_by_width<float, 1, BACKWARD>(a);
  return vec ? norm_by_width<__nv_bfloat16, vec16<__nv_bfloat16>(), BACKWARD>(a) : norm_by_width<__nv_bfloat16, 1, BACKWARD>(a);
}

int norm_check(int32_t rows, int32_t d, int64_t ldx, int32_t dtype, int32_t w_dtype) {
  if (rows < 0 || d < 1 || ldx < d) return GROUTER_ERR_INVALID_ARG;
  if ((dtype != GROUTER_BF16 && dtype != GROUTER_F32) || (w_dtype != GROUTER_BF16 && w_dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  // the row counters of the resident blocks step past the last row by up to one grid
  return d > NORM_MAX_D || rows > INT32_MAX - (1 << 20) ? GROUTER_ERR_UNSUPPORTED : GROUTER_OK;
}

}  // namespace
}  // namespace grouter

using namespace grouter;

extern "C" {

int grouter_layernorm_fwd(const void* x, int64_t ldx, const void* w, const void* b, int32_t rows, int32_t d, int32_t dtype, int32_t w_dtype,
                          float eps, void* y, float* mean, float* rstd, void* stream) {
  if (!w || !(eps >= 0.f) || (rows > 0 && (!x || !y))) return GROUTER_ERR_INVALID_ARG;
  if (const int e = norm_check(rows, d, ldx, dtype, w_dtype)) return e;
  const size_t el = dtype == GROUTER_F32 ? 4 : 2, wl = w_dtype == GROUTER_F32 ? 4 : 2;
  if (!aligned_to(x, el) || !aligned_to(y, el) || !aligned_to(w, wl) || !aligned_to(b, wl) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
    return GROUTER_ERR_MISALIGNED;
  if (rows == 0) return GROUTER_OK;
  NormArgs a{};
  a.x = x; a.ldx = ldx; a.w = w; a.b = b; a.w_f32 = w_dtype == GROUTER_F32; a.rows = rows; a.d = d; a.eps = eps;
  a.y = y; a.mean_out = mean; a.rstd_out = rstd; a.st = static_cast<cudaStream_t>(stream);
  return norm_dispatch<false>(a, dtype) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

size_t grouter_layernorm_bwd_workspace_bytes(int32_t rows, int32_t d) {
  if (rows < 0 || d < 1 || d > NORM_MAX_D) return 0;
  return (size_t)(rows ? norm_backward_blocks(rows, d) : 1) * 2 * d * sizeof(float);
}

int grouter_layernorm_bwd(const void* dy, const void* x, int64_t ldx, const void* w, const float* mean, const float* rstd, int32_t rows,
                          int32_t d, int32_t dtype, int32_t w_dtype, void* dx, float* dw, float* db, void* workspace, void* stream) {
  if (!w || !dw || (rows > 0 && (!dy || !x || !mean || !rstd || !dx || !workspace))) return GROUTER_ERR_INVALID_ARG;
  if (const int e = norm_check(rows, d, ldx, dtype, w_dtype)) return e;
  const size_t el = dtype == GROUTER_F32 ? 4 : 2, wl = w_dtype == GROUTER_F32 ? 4 : 2;
  if (!aligned_to(x, el) || !aligned_to(dy, el) || !aligned_to(dx, el) || !aligned_to(w, wl) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) ||
      !aligned_to(dw, 4) || !aligned_to(db, 4) || !aligned_to(workspace, 16))
    return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {        // sums over no rows
    if (cudaMemsetAsync(dw, 0, (size_t)d * 4, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    if (db && cudaMemsetAsync(db, 0, (size_t)d * 4, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    return GROUTER_OK;
  }
  NormArgs a{};
  a.dy = dy; a.x = x; a.ldx = ldx; a.w = w; a.w_f32 = w_dtype == GROUTER_F32; a.mean_in = mean; a.rstd_in = rstd; a.rows = rows; a.d = d;
  a.dx = dx; a.dw = dw; a.db = db; a.partial = static_cast<float*>(workspace); a.st = st;
  return norm_dispatch<true>(a, dtype) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
