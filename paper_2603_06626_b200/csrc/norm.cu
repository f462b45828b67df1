// Layer norm over the rows of a matrix, forward and backward.
//
//   forward    mean_t = (1/d) sum_j x_tj     rstd_t = ((1/d) sum_j (x_tj - mean_t)^2 + eps)^(-1/2)
//              y_tj = (x_tj - mean_t) rstd_t w_j + b_j
//   backward   h = (x - mean) rstd,  g = dy w
//              dx_tj = rstd_t (g_tj - (1/d) sum_i g_ti - h_tj (1/d) sum_i g_ti h_ti)
//              dw_j = sum_t dy_tj h_tj       db_j = sum_t dy_tj
//
// Both passes touch every element once and are bound by HBM, but only if they are lean: at 6.4 TB/s an SM has some 20 (forward)
// and 30 (backward) instruction slots for an element of bf16, so the arithmetic is done two elements to an instruction (f32x2).
// Sums are taken in fp32, the variance from the centred values (never as a difference of large sums).
// Measured on a B200 whose plain copy runs at 6.46 TB/s: forward 32768 x 4096 bf16 84 us (6.4 TB/s), 65536 x 512 22-25 us (6.1-5.3),
// 8192 x 16384 85 us (6.3);  backward with both kernels 16384 x 4096 bf16 74 us (5.4), 16384 x 2048 43 us (4.7), 8192 x 4096 f32 74 us
// (5.4), 8192 x 16384 f32 299 us (5.4) and bf16 202 us (4.0: 1024 threads a row, one row an SM).  Rows that are not 16-byte aligned go
// by pairs, or by single elements where even those do not fit: 16384 x 4094 bf16 55 us forward, 100 us backward, 16384 x 4095 88
// and 117 us.  Wider than 8192 such rows spill registers in the backward pass (160 to 192 bytes a thread): 8192 x 16383 bf16 395 us.
//   Forward: a row lies in the registers of as many lanes (a quarter of a warp to 32 warps) as hold it in a few accesses each, as it
//     was loaded; nothing is kept from row to row.
//   Backward: the running dw and db of a column have to stay with one thread, so a row is spread over enough threads for 16
//     elements each (eight for a row of 128: 262144 x 128 bf16 39 us, with a warp 87); blocks are resident and walk over the rows (the
//     coming ones on their way into shared memory), every cluster of them writes one partial row, and a second small kernel adds
//     those up in a fixed order (bit-reproducible, no atomics).
#include <cooperative_groups.h>

#include <algorithm>

#include "norm.cuh"

namespace grouter {

constexpr int NORM_MAX_D = 16384;

// ---- forward: LANES threads a row, NP accesses of VE elements each ----
__host__ __device__ constexpr int norm_forward_threads(int lanes) { return lanes <= 32 ? 128 : lanes; }

template <typename T, typename W, int VE, int NP, int LANES>
__global__ void __launch_bounds__(norm_forward_threads(LANES)) norm_forward_kernel(const T* __restrict__ x, int64_t ldx, const W* __restrict__ w,
                                                                                const W* __restrict__ b, int rows, int d, float eps,
                                                                                T* __restrict__ y, float* __restrict__ mean_out,
                                                                                float* __restrict__ rstd_out) {
  constexpr int RPB = norm_forward_threads(LANES) / LANES;
  __shared__ float red[2 * 32];
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LANES;
  const int at = threadIdx.x & (LANES - 1);
  if (LANES >= 32 && row >= rows) return;  // whole warps, and whole blocks where a row has several
  // A row that is not there stays for the sums of those beside it in the warp, without elements (end), its mean a plain 0: dividing by
  // a d of 0 sent such lanes down the slow paths of quotient and root (1 x 128 bf16: 1.9 -> 2.1 us).
  const int end = LANES >= 32 || row < rows ? d : 0;
  const T* xr = x + row * ldx;
  Pack<T, VE> p[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int c = (n * LANES + at) * VE;
    if (c < end) p[n] = ld_pack<T, VE>(xr + c);
  }
  const float inv_d = 1.f / (float)d;
  int half = 0;
  float s[1] = {0.f};
  if constexpr (VE > 1) {
    float2 s2 = both(0.f);
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if ((n * LANES + at) * VE < end) {
#pragma unroll
        for (int i = 0; i < VE; i += 2) s2 = add2(s2, pair_at(p, (n * VE + i) / 2));
      }
    s[0] = s2.x + s2.y;
  } else {
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if (n * LANES + at < end) s[0] += to_f32(p[n].v[0]);
  }
  row_sums<LANES, 1>(s, red, half);
  const float mean = s[0] * inv_d;
  float q[1] = {0.f};
  if constexpr (VE > 1) {
    float2 q2 = both(0.f);
    const float2 m2 = both(-mean);
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if ((n * LANES + at) * VE < end) {
#pragma unroll
        for (int i = 0; i < VE; i += 2) {
          const float2 c2 = add2(pair_at(p, (n * VE + i) / 2), m2);
          q2 = fma2(c2, c2, q2);
        }
      }
    q[0] = q2.x + q2.y;
  } else {
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if (n * LANES + at < end) {
        const float c1 = to_f32(p[n].v[0]) - mean;
        q[0] += c1 * c1;
      }
  }
  row_sums<LANES, 1>(q, red, half);
  const float rstd = 1.f / sqrtf(q[0] * inv_d + eps);
  T* yr = y + row * d;
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int c = (n * LANES + at) * VE;
    if (c < end) {
      float wl[VE], bl[VE], o[VE];
      load_weights<W, VE>(w, c, wl);
      if (b != nullptr) {
        load_weights<W, VE>(b, c, bl);
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i) bl[i] = 0.f;
      }
      if constexpr (VE > 1) {
#pragma unroll
        for (int i = 0; i < VE; i += 2) {
          const float2 h = mul2(add2(pair_at(p, (n * VE + i) / 2), both(-mean)), both(rstd));
          const float2 v = fma2(h, make_float2(wl[i], wl[i + 1]), make_float2(bl[i], bl[i + 1]));
          o[i] = v.x;
          o[i + 1] = v.y;
        }
      } else {
        o[0] = (to_f32(p[n].v[0]) - mean) * rstd * wl[0] + bl[0];
      }
      st_pack<T, VE>(yr + c, o);
    }
  }
  if (at == 0 && row < rows) {
    if (mean_out) mean_out[row] = mean;
    if (rstd_out) rstd_out[row] = rstd;
  }
}

// ---- backward: TPR threads a row, NORM_EPT elements each ----
constexpr int NORM_EPT = 16;
__host__ __device__ constexpr int norm_backward_threads(int tpr) { return tpr <= 32 ? 256 : tpr; }
__host__ __device__ constexpr int norm_backward_per_sm(int tpr) { return tpr >= 512 ? 1 : 512 / norm_backward_threads(tpr); }
// Rows (x and dy) that a block has on their way or in use: what keeps HBM busy (rows held one ahead in registers were 32 KB an SM
// and 3.6 TB/s).  As many as shared memory takes: an SM holds 512 threads' rows, 1024 for the widest.
__host__ __device__ constexpr int norm_ring(int bytes, int tpr) { return tpr == 1024 ? (bytes == 2 ? 3 : 1) : bytes == 2 ? 4 : 3; }

// Every thread copies its own elements of the coming rows into shared memory and reads back only those, so the ring needs no
// barrier: the one barrier a row is that of its two sums.  Rows that are not 16-byte aligned: plain loads, no ring
// (one of 4-byte copies: 8192 x 4095 f32 78 -> 91 us).
template <typename T, typename W, int VE, int TPR>
__global__ void __launch_bounds__(norm_backward_threads(TPR), norm_backward_per_sm(TPR))
norm_backward_kernel(const T* __restrict__ dy, const T* __restrict__ x, int64_t ldx, const W* __restrict__ w, const float* __restrict__ mean_in,
                     const float* __restrict__ rstd_in, int rows, int d, T* __restrict__ dx, float* __restrict__ partial) {
  constexpr int NV = NORM_EPT / VE, PAIRS = NORM_EPT / 2;
  constexpr int THREADS = norm_backward_threads(TPR), RPB = THREADS / TPR;
  constexpr bool RING = VE * sizeof(T) == 16;
  constexpr int S = norm_ring(sizeof(T), TPR);
  constexpr bool HOLD = TPR < 1024;     // the weights stay in registers (1024 threads have 64 each: there they are read from L1)
  extern __shared__ uint4 s_ring[];     // RING: [S][x, dy][NV][THREADS]; at the end this block's columns, [dw | db]
  __shared__ float red[2 * 2 * 32];
  const int lane = threadIdx.x & (TPR - 1);
  const int sub = threadIdx.x / TPR;
  const float inv_d = 1.f / (float)d;
  // a thread's elements in pairs: pair j holds elements 2j and 2j + 1 of its [NV][VE]; columns beyond d hold zeros throughout
  auto weights = [&](float2 (&f)[PAIRS]) {
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      float t[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) t[i] = 0.f;
      const int c = (n * TPR + lane) * VE;
      if (c < d) load_weights<W, VE>(w, c, t);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const int k = n * VE + i;
        if (k & 1) f[k / 2].y = t[i];
        else f[k / 2].x = t[i];
      }
    }
  };
  float2 wv[PAIRS], aw[PAIRS], ab[PAIRS];
  if constexpr (HOLD) weights(wv);
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) aw[j] = ab[j] = both(0.f);

  auto slot = [&](int s, int which, int n) { return s_ring + ((s * 2 + which) * NV + n) * THREADS + threadIdx.x; };
  auto fetch = [&](int64_t r, int s) {
    if (r < rows) {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const int c = (n * TPR + lane) * VE;
        if (c < d) {
          copy16_async(slot(s, 0, n), x + r * ldx + c);
          copy16_async(slot(s, 1, n), dy + r * d + c);
        }
      }
    }
    copies_commit();
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  const int64_t step = (int64_t)gridDim.x * RPB;
  float nmean = 0.f, nrstd = 0.f;
  auto stats = [&](int64_t r) {
    if (r < rows) {
      nmean = __ldg(mean_in + r);
      nrstd = __ldg(rstd_in + r);
    }
  };
  stats(row);
  if constexpr (RING) {
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if ((n * TPR + lane) * VE >= d)
        for (int s = 0; s < S; ++s) *slot(s, 0, n) = *slot(s, 1, n) = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(row + s * step, s);
  }
  int half = 0, s_at = 0;
  // rows that share a warp stay together for their sums: those past the last row hold zeros
  const int behind = TPR < 32 ? sub & (32 / TPR - 1) : 0;
  for (; row - behind < rows; row += step) {
    const bool live = TPR >= 32 || row < rows;
    const float mean = live ? nmean : 0.f, rstd = live ? nrstd : 0.f;
    stats(row + step);
    Pack<T, VE> px[NV], pg[NV];
    auto take = [&]() {                 // this row's elements
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        if constexpr (RING) {
          const uint4 zeros = make_uint4(0u, 0u, 0u, 0u);
          *reinterpret_cast<uint4*>(&px[n]) = live ? *slot(s_at, 0, n) : zeros;
          *reinterpret_cast<uint4*>(&pg[n]) = live ? *slot(s_at, 1, n) : zeros;
        } else {
          const int c = (n * TPR + lane) * VE;
#pragma unroll
          for (int i = 0; i < VE; ++i) px[n].v[i] = pg[n].v[i] = from_f32<T>(0.f);
          if (c < d && live) {
            px[n] = ld_pack<T, VE>(x + row * ldx + c);
            pg[n] = ld_pack<T, VE>(dy + row * d + c);
          }
        }
      }
    };
    if constexpr (RING) copies_wait<S - 1>();
    take();
    if constexpr (!HOLD) weights(wv);
    // with 128 registers a thread the centred row and dy stay where they are; with 64 they are read again after the sums
    float2 xc[PAIRS], g0[PAIRS];
    auto open = [&](int j) {
      g0[j] = pair_at(pg, j);
      xc[j] = add2(pair_at(px, j), both(-mean));
    };
    float2 s1 = both(0.f), s2 = both(0.f);            // sums of g and of g (x - mean)
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      open(j);
      aw[j] = fma2(g0[j], mul2(xc[j], both(rstd)), aw[j]);
      ab[j] = add2(ab[j], g0[j]);
      const float2 g = mul2(g0[j], wv[j]);
      s1 = add2(s1, g);
      s2 = fma2(g, xc[j], s2);
    }
    float s[2] = {s1.x + s1.y, s2.x + s2.y};
    row_sums<TPR, 2>(s, red, half);
    // dx = rstd g w - rstd mean(g) - (x - mean) rstd^3 mean(g (x - mean))
    const float2 r = both(rstd), c1 = both(-s[0] * inv_d * rstd), c2 = both(-s[1] * inv_d * rstd * rstd * rstd);
    if constexpr (!HOLD) {
      asm volatile("" ::: "memory");
      weights(wv);
      if constexpr (RING) take();
      else forget<T, VE, NV>(px), forget<T, VE, NV>(pg);
    }
    T* dr = dx + row * d;
    float o[NORM_EPT];
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      if constexpr (!HOLD) open(j);
      const float2 v = fma2(xc[j], c2, fma2(mul2(g0[j], wv[j]), r, c1));
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
  cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
  const int CL = (int)cl.num_blocks();
  float* pw = partial + (int64_t)(blockIdx.x / CL) * 2 * d;
  // this thread's columns, VE at a time (one float at a time, a block of 32 short rows: eight lanes to a bank; 1 x 128 bf16 4.1 -> 3.4 us,
  // 3000 x 2048 23.8 -> 14.6)
  auto put_columns = [&](float* row_of) {
    if constexpr (!HOLD && sizeof(T) == 4) {       // f32 rows of 1024 threads: one by one (8192 x 16384 295 us, 16 bytes at a time 301)
#pragma unroll
      for (int k = 0; k < NORM_EPT; ++k) {
        const int c = ((k / VE) * TPR + lane) * VE + k % VE;
        if (c < d) {
          row_of[c] = k & 1 ? aw[k / 2].y : aw[k / 2].x;
          row_of[d + c] = k & 1 ? ab[k / 2].y : ab[k / 2].x;
        }
      }
      return;
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + lane) * VE;
      if (c < d) {
        store_floats<VE>(row_of + c, [&](int i) { return (n * VE + i) & 1 ? aw[(n * VE + i) / 2].y : aw[(n * VE + i) / 2].x; });
        store_floats<VE>(row_of + d + c, [&](int i) { return (n * VE + i) & 1 ? ab[(n * VE + i) / 2].y : ab[(n * VE + i) / 2].x; });
      }
    }
  };
  if (RPB == 1 && CL == 1) {             // nobody to add up with: no cluster, no barrier (1 x 1024: 5.5 -> 3.6 us)
    put_columns(pw);
    return;
  }
  // this block's columns, [dw | db], take the ring's place (nothing is on its way into it any more)
  float* cols = reinterpret_cast<float*>(s_ring);
  __syncthreads();
  put_columns(cols + sub * 2 * d);       // each of the rows that the block works on at a time has its own
  if constexpr (RPB > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * d; c += THREADS) {
      float a = cols[c];
#pragma unroll
      for (int r = 1; r < RPB; ++r) a += cols[r * 2 * d + c];
      if (CL == 1) pw[c] = a;
      else cols[c] = a;
    }
    if (CL == 1) return;
  }
  // the cluster's blocks add up a share of the columns each, in rank order, into one partial row
  cl.sync();
  for (int c = (int)cl.block_rank() * THREADS + threadIdx.x; c < 2 * d; c += CL * THREADS) {
    float a = 0.f;
    for (int r = 0; r < CL; ++r) a += cl.map_shared_rank(cols, r)[c];
    pw[c] = a;
  }
  cl.sync();                            // nobody leaves while its columns are read
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
  let_next_kernel_start();
  if (c < cols) {
#pragma unroll 16
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

// Threads that hold a row of d elements in the backward pass.
int norm_tpr(int d) {
  int tpr = 8;
  while (tpr * NORM_EPT < d) tpr *= 2;
  return tpr;
}

// Blocks of the backward pass: enough to fill the GPU, no more than there are rows for, and whole clusters: neighbouring blocks
// that add up their columns through each other's shared memory and leave one partial row.
//   A row a block: the partial rows are as large as the problem, so eight blocks join (1000 x 1024: 18 -> 9.6 us, in pairs 15), or
//     two of the larger ones, of which an SM holds few; very few rows do without (20 x 4096: 8.0 us, in pairs 10).
//   Many rows a block: pairs (16384 x 2048: 47 -> 44 us, 8192 x 16384 f32: 367 -> 298; clusters of eight leave places for blocks empty:
//     55 us, 65536 x 1024 73 in pairs and 97 in eights); one warp a row gains nothing (65536 x 512: 40 us either way),
//     and rows without a ring lose (16384 x 2047 bf16: 59 -> 64, 16384 x 4095 116 -> 119, 8192 x 4095 f32 76 -> 78).
struct NormGrid {
  int blocks, cluster;
  int parts() const { return blocks / cluster; }      // partial rows they leave
};
NormGrid norm_backward_grid(int rows, int d, bool ring) {
  const int tpr = norm_tpr(d), rpb = norm_backward_threads(tpr) / tpr;
  const int want = (rows + rpb - 1) / rpb, cap = current_sms() * norm_backward_per_sm(tpr);
  NormGrid g{want < cap ? want : cap, 1};
  if (want <= cap) g.cluster = want < 64 ? 1 : tpr <= 128 ? 8 : 2;
  else if (ring && tpr >= 64 && want >= 8 * cap) g.cluster = 2;
  g.blocks -= g.blocks % g.cluster;
  return g;
}

template <typename T, typename W, int VE, int NP, int LANES>
cudaError_t forward_launch(const NormArgs& a) {
  constexpr int THREADS = norm_forward_threads(LANES), RPB = THREADS / LANES;
  norm_forward_kernel<T, W, VE, NP, LANES><<<(a.rows + RPB - 1) / RPB, THREADS, 0, a.st>>>(
      static_cast<const T*>(a.x), a.ldx, static_cast<const W*>(a.w), static_cast<const W*>(a.b), a.rows, a.d, a.eps, static_cast<T*>(a.y), a.mean_out,
      a.rstd_out);
  return cudaGetLastError();
}

// Up to FEW accesses a lane while a quarter of a warp holds a row, then more lanes; a warp's lanes then take up to MOST, more warps
// follow up to LAST lanes, those take twice MOST before warps follow up to 16, and what is still needed of both.
template <typename T, typename W, int VE, int MOST, int FEW, int LAST, int NP = 1, int LANES = 8>
cudaError_t forward_spread(const NormArgs& a) {
  constexpr int HOLDS = NP * LANES * VE;
  if constexpr (HOLDS < NORM_MAX_D) {
    if (a.d > HOLDS) {
      constexpr bool more = NP < FEW || (LANES >= 32 && (NP < MOST || (LANES == LAST && NP < 2 * MOST) || (LANES == 512 && NP < 16)));
      if constexpr (more) return forward_spread<T, W, VE, MOST, FEW, LAST, 2 * NP, LANES>(a);
      else return forward_spread<T, W, VE, MOST, FEW, LAST, NP, 2 * LANES>(a);
    }
  }
  return forward_launch<T, W, VE, NP, LANES>(a);
}

// Four 16-byte accesses a lane (16384 x 4096 bf16: 44.6 us, with sixteen 52.3, with two 52.7; 65536 x 128 7.9 us, with one access of 16
// lanes 9.4, of a warp 16), and fewer, in more lanes, where the whole matrix is small and the time is that of a row (1 x 4096: 2.6
// against 3.0 us, 1024 x 2048 3.3 against 4.0, but 1024 x 4096 5.3 against 4.3); eight of the smaller ones (16384 x 4094: 54 us, with
// four 79).
// The widest rows take eight accesses of eight warps before more warps (8192 x 16384 bf16: 107 us, four of sixteen warps 129; 8192 x 12288 84 and
// 104; but 140 x 16384 5.8 and 5.1), large matrices of single bf16 under f32 weights sixteen (16384 x 2047: 42 us, with eight 44, 16384 x 4095
// 85.5 and 90; but 1000 x 4095 10.6 and 8.6, and under bf16 weights 16384 x 2047 44.5 and 42).
constexpr int64_t NORM_SMALL = 1 << 21;
template <typename T, typename W, int VE>
cudaError_t forward_by_width(const NormArgs& a) {
  const int64_t size = (int64_t)a.rows * a.d;
  if constexpr (VE * sizeof(T) == 2 && sizeof(W) == 4) {
    return size <= 8 * NORM_SMALL ? forward_spread<T, W, VE, 8, 4, 512>(a) : forward_spread<T, W, VE, 16, 4, 512>(a);
  } else if constexpr (VE * sizeof(T) < 16) {
    return forward_spread<T, W, VE, 8, 4, 512>(a);
  } else {
    if (size <= NORM_SMALL) return forward_spread<T, W, VE, 2, 1, 512>(a);
    return size <= 2 * NORM_SMALL ? forward_spread<T, W, VE, 4, 4, 512>(a) : forward_spread<T, W, VE, 4, 4, 256>(a);
  }
}

template <typename T, typename W, int VE, int TPR>
cudaError_t backward_launch(const NormArgs& a) {
  const NormGrid g = norm_backward_grid(a.rows, a.d, VE == vec16<T>());
  constexpr int threads = norm_backward_threads(TPR), ring = VE == vec16<T>() ? norm_ring(sizeof(T), TPR) * 2 * (NORM_EPT / VE) * threads * 16 : 0;
  constexpr int cols = 2 * threads * NORM_EPT * (int)sizeof(float);
  constexpr int smem = ring > cols ? ring : cols;      // up to 192 KB
  auto kern = norm_backward_kernel<T, W, VE, TPR>;
  static bool configured[64] = {};                     // the opt-in is a per-device setting
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(g.blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = a.st;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = g.cluster;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = g.cluster > 1 ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, static_cast<const T*>(a.dy), static_cast<const T*>(a.x), a.ldx, static_cast<const W*>(a.w),
                                           a.mean_in, a.rstd_in, a.rows, a.d, static_cast<T*>(a.dx), a.partial);
  if (e != cudaSuccess) return e;
  return launch_sum_rows(a.partial, g.parts(), 2 * a.d, a.dw, a.d, a.db, a.st);
}

template <typename T, typename W, int VE>
cudaError_t backward_by_width(const NormArgs& a) {
  switch (norm_tpr(a.d)) {
    case 8: return backward_launch<T, W, VE, 8>(a);
    case 16: return backward_launch<T, W, VE, 16>(a);
    case 32: return backward_launch<T, W, VE, 32>(a);
    case 64: return backward_launch<T, W, VE, 64>(a);
    case 128: return backward_launch<T, W, VE, 128>(a);
    case 256: return backward_launch<T, W, VE, 256>(a);
    case 512: return backward_launch<T, W, VE, 512>(a);
    default: return backward_launch<T, W, VE, 1024>(a);
  }
}

template <bool BACKWARD, typename T, typename W, int VE>
cudaError_t norm_by_width(const NormArgs& a) {
  if constexpr (BACKWARD) return backward_by_width<T, W, VE>(a);
  else return forward_by_width<T, W, VE>(a);
}
template <bool BACKWARD, typename T, int VE>
cudaError_t norm_by_weights(const NormArgs& a) {
  return a.w_f32 ? norm_by_width<BACKWARD, T, float, VE>(a) : norm_by_width<BACKWARD, T, __nv_bfloat16, VE>(a);
}
template <bool BACKWARD, typename T>
cudaError_t norm_by_type(const NormArgs& a) {
  // accesses of VE elements where every row of every activation and the weights start on a boundary of them
  auto fits = [&](int ve) {
    const size_t b = ve * sizeof(T), wb = std::min<size_t>(ve * (a.w_f32 ? 4 : 2), 16);
    return a.d % ve == 0 && a.ldx % ve == 0 && aligned_to(a.x, b) && aligned_to(BACKWARD ? a.dy : a.y, b) && (!BACKWARD || aligned_to(a.dx, b)) &&
           aligned_to(a.w, wb) && aligned_to(a.b, wb);
  };
  if (fits(vec16<T>())) return norm_by_weights<BACKWARD, T, vec16<T>()>(a);
  if (fits(2)) return norm_by_weights<BACKWARD, T, 2>(a);
  return norm_by_weights<BACKWARD, T, 1>(a);
}
template <bool BACKWARD>
cudaError_t norm_dispatch(const NormArgs& a, int dtype) {
  return dtype == GROUTER_F32 ? norm_by_type<BACKWARD, float>(a) : norm_by_type<BACKWARD, __nv_bfloat16>(a);
}

int norm_check(int32_t rows, int32_t d, int64_t ldx, int32_t dtype, int32_t w_dtype) {
  if (rows < 0 || d < 1 || ldx < d) return GROUTER_ERR_INVALID_ARG;
  if ((dtype != GROUTER_BF16 && dtype != GROUTER_F32) || (w_dtype != GROUTER_BF16 && w_dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  // rows are rounded up to whole blocks in 32 bits
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
  if (norm_check(rows, d, d, GROUTER_BF16, GROUTER_BF16) != GROUTER_OK) return 0;
  // alignment is not known here: as many partial rows as rows without a ring leave
  return (size_t)std::max(norm_backward_grid(rows, d, false).parts(), 1) * 2 * d * sizeof(float);
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
