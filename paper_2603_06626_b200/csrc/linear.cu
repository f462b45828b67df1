// Linear layer with bias, activation and residual in the epilogue of its product, and its gradients.
//
//   forward    z = x W^T + b       y = act(z) + r                                    x [T,K], W [N,K], y, z, r [T,N]
//   backward   dz = dy act'(z)     dx = dz W      dW = dz^T x      db = sum_t dz      (the residual's gradient is dy itself)
//
// The products run on the CTA-pair tcgen05 core of the grouped products (gemm.cu, MODE_LINEAR / MODE_DENSE) or, for few tokens, on
// the kernel of linear_small.cu: bf16 operands, fp32 accumulators; bias, activation and residual are applied in fp32 on the
// accumulator and rounded once.  Bound by the tensor cores: 32768 x 4096 x 1536 with SiLU and both outputs takes 312-353 us, 1.32-1.17
// PFLOP/s as the GPU goes from rested to its power limit; without the epilogue 288-328, as long as a library's product of these
// sizes (292-328).  8192 x 8192 x 8192 plain: 1.48-1.26 PFLOP/s, 8 to 9 % behind the library's 1.63-1.38.
// dz is rounded to bf16, the type the tensor cores take it in; db is summed from the unrounded values.  One pass over dy and
// z writes dz and the partial column sums; without an activation dz is dy and the pass only sums (or is left out).
// dW's output matrix is often too small to give every CTA pair a tile: its contraction over the tokens is then cut into
// pieces, stored as fp32 matrices and added up by a last pass in a fixed order.
#include "act.cuh"
#include "vec.cuh"

namespace grouter {

constexpr int DZ_THREADS = 256;
constexpr int DZ_COLS = 256;            // columns of a block: 32 threads of 8
constexpr int DZ_LANES = DZ_THREADS * 8 / DZ_COLS;      // rows it works on at a time

// dz = dy act'(z) (WRITE), and the column sums of this block's rows (SUM) as row blockIdx.y of `partial` [gridDim.y][N].  A thread has
// DZ_AHEAD rows' loads on their way at a time.
template <int ACT, bool WRITE, bool SUM>
__global__ void __launch_bounds__(DZ_THREADS) linear_dz_kernel(const __nv_bfloat16* __restrict__ dy, const __nv_bfloat16* __restrict__ z, int T,
                                                               int N, __nv_bfloat16* __restrict__ dz, float* __restrict__ partial) {
  constexpr int DZ_AHEAD = 4;
  __shared__ float s_sum[SUM ? DZ_LANES : 1][DZ_COLS + 1];
  const int ct = threadIdx.x & 31, rl = threadIdx.x >> 5;
  const int c = blockIdx.x * DZ_COLS + ct * 8;
  float2 acc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = both(0.f);
  after_previous_kernel();
  if (c < N) {
    const int64_t step = (int64_t)gridDim.y * DZ_LANES;
    for (int64_t t0 = (int64_t)blockIdx.y * DZ_LANES + rl; t0 < T; t0 += step * DZ_AHEAD) {
      Pack<__nv_bfloat16, 8> g[DZ_AHEAD], q[DZ_AHEAD];
#pragma unroll
      for (int u = 0; u < DZ_AHEAD; ++u) {
        const int64_t t = t0 + u * step;
        if (t < T) {
          g[u] = ld_pack<__nv_bfloat16, 8>(dy + t * N + c);
          if (ACT != GROUTER_ACT_NONE) q[u] = ld_pack<__nv_bfloat16, 8>(z + t * N + c);
        }
      }
#pragma unroll
      for (int u = 0; u < DZ_AHEAD; ++u) {
        const int64_t t = t0 + u * step;
        if (t < T) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            float2 w = pair_at(g, 4 * u + i / 2);
            if (ACT != GROUTER_ACT_NONE) w = act_back2<ACT>(w, pair_at(q, 4 * u + i / 2));
            if (SUM) acc[i / 2] = add2(acc[i / 2], w);
            v[i] = w.x;
            v[i + 1] = w.y;
          }
          if (WRITE) st_pack<__nv_bfloat16, 8>(dz + t * N + c, v);
        }
      }
    }
  }
  let_next_kernel_start();
  if constexpr (SUM) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s_sum[rl][ct + 64 * i] = acc[i].x;
      s_sum[rl][ct + 64 * i + 32] = acc[i].y;
    }
    __syncthreads();
    for (int q = threadIdx.x; q < DZ_COLS; q += DZ_THREADS) {
      float a = 0.f;
#pragma unroll
      for (int l = 0; l < DZ_LANES; ++l) a += s_sum[l][q];
      const int col = blockIdx.x * DZ_COLS + (q & 31) * 8 + (q >> 5);
      if (col < N) partial[(int64_t)blockIdx.y * N + col] = a;
    }
  }
}

// out = sum of `pieces` matrices of n4 x 4 values, in order.
template <typename T>
__global__ void __launch_bounds__(256) sum_pieces_kernel(const float* __restrict__ in, int pieces, int64_t n4, T* __restrict__ out) {
  after_previous_kernel();
  let_next_kernel_start();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    float4 a = __ldcs(reinterpret_cast<const float4*>(in) + i);
    for (int q = 1; q < pieces; ++q) {
      const float4 b = __ldcs(reinterpret_cast<const float4*>(in) + q * n4 + i);
      a.x += b.x;
      a.y += b.y;
      a.z += b.z;
      a.w += b.w;
    }
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(out)[i] = a;
    } else {
      uint2 r;
      *reinterpret_cast<__nv_bfloat162*>(&r.x) = __floats2bfloat162_rn(a.x, a.y);
      *reinterpret_cast<__nv_bfloat162*>(&r.y) = __floats2bfloat162_rn(a.z, a.w);
      reinterpret_cast<uint2*>(out)[i] = r;
    }
  }
}

namespace {

inline int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Pieces the contraction of dW over T tokens is cut into.  Cost in k-steps (64 tokens of one 256 x 256 tile): rounds of the CTA
// pairs times steps a round; a piece costs writing and reading back its matrix, about a third of a step a tile at L2's pace.
int dw_pieces(int T, int K, int N) {
  const int pairs = current_sms() / 2, tiles = cdiv(N, 256) * cdiv(K, 256), steps = cdiv(T, 64);
  int best = 1;
  float best_cost = 0.f;
  for (int s = 1; s <= 16 && (s == 1 || steps / s >= 8); ++s) {
    const float cost = (float)cdiv((int64_t)tiles * s, pairs > 0 ? pairs : 1) * cdiv(steps, s) + (s > 1 ? 0.33f * s * tiles : 0.f);
    if (s == 1 || cost < best_cost) {
      best = s;
      best_cost = cost;
    }
  }
  return best;
}
inline int dw_chunk(int T, int pieces) { return cdiv(cdiv(T, 64), pieces) * 64; }

// Row blocks of the dz pass: about six blocks an SM over all columns, at least four rows for every thread.
int dz_row_blocks(int T, int N) {
  const int cols = cdiv(N, DZ_COLS);
  const int want = cdiv((int64_t)current_sms() * 6, cols), most = cdiv(T, DZ_LANES * 4);
  const int r = want < most ? want : most;
  return r < 1 ? 1 : r;
}

struct LinearWorkspace {
  size_t dz, sums, pieces, bytes;
};
LinearWorkspace linear_workspace(int T, int K, int N, int act) {
  LinearWorkspace w{};
  w.dz = 0;
  w.sums = w.dz + (act == GROUTER_ACT_NONE ? 0 : up256((size_t)T * N * 2));
  w.pieces = w.sums + up256((size_t)dz_row_blocks(T, N) * N * 4);
  const int s = dw_pieces(T, K, N);
  w.bytes = w.pieces + (s > 1 ? up256((size_t)s * N * K * 4) : 0) + 256;
  return w;
}

template <int ACT>
cudaError_t launch_dz_act(const void* dy, const void* z, int T, int N, void* dz, float* partial, dim3 grid, cudaStream_t st) {
  const __nv_bfloat16 *g = static_cast<const __nv_bfloat16*>(dy), *p = static_cast<const __nv_bfloat16*>(z);
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(dz);
  if (partial) return launch_dependent(linear_dz_kernel<ACT, ACT != GROUTER_ACT_NONE, true>, grid, dim3(DZ_THREADS), 0, st, g, p, T, N, o, partial);
  if constexpr (ACT != GROUTER_ACT_NONE)      // without an activation there is nothing to write either
    return launch_dependent(linear_dz_kernel<ACT, true, false>, grid, dim3(DZ_THREADS), 0, st, g, p, T, N, o, partial);
  return cudaSuccess;
}
cudaError_t launch_dz(int act, const void* dy, const void* z, int T, int N, void* dz, float* partial, int row_blocks, cudaStream_t st) {
  const dim3 grid(cdiv(N, DZ_COLS), row_blocks);
  switch (act) {
    case GROUTER_ACT_RELU: return launch_dz_act<GROUTER_ACT_RELU>(dy, z, T, N, dz, partial, grid, st);
    case GROUTER_ACT_SILU: return launch_dz_act<GROUTER_ACT_SILU>(dy, z, T, N, dz, partial, grid, st);
    case GROUTER_ACT_GELU: return launch_dz_act<GROUTER_ACT_GELU>(dy, z, T, N, dz, partial, grid, st);
    default: return launch_dz_act<GROUTER_ACT_NONE>(dy, z, T, N, dz, partial, grid, st);
  }
}

// y or dx: the CTA-pair core, or the kernel for few tokens.  Both sides in rounds of the machine times 64-deep steps a round,
// measured over T = 1 .. 4096 and weights of 128 x 128 to 4096 x 4096: a step takes 0.33 us on 256 x 256 tiles (5.7 us around them)
// and 0.45 us on two 128 x 128 tiles an SM (7.5 us around them, and as much again for every further round); up to 64 tokens the
// tiles are narrower and their kernel ahead throughout (one token, 4096 x 4096: 8.4 against 38 us; 128 tokens, 512 -> 4096: 9.8
// against 8.9; 512 tokens, 4096 x 4096: 23.5 against 26.8; 1024: 34.5 against 28.4).
cudaError_t launch_product(const LinearGemm& g, cudaStream_t st) {
  const int sms = current_sms(), splits = linear_small_splits(g.M, g.N, g.K), steps = cdiv(g.K, 64);
  const int big_rounds = cdiv((int64_t)cdiv(g.M, 256) * cdiv(g.N, 256), sms / 2 > 0 ? sms / 2 : 1);
  const int small_rounds = cdiv((int64_t)cdiv(g.M, 128) * cdiv(g.N, 128) * splits, 2 * sms > 0 ? 2 * sms : 1);
  const float big = 5.7f + 0.33f * big_rounds * steps, small = small_rounds * (7.5f + 0.45f * cdiv(steps, splits));
  const bool fits = cdiv(g.M, 128) <= 65535;      // its grid has the token tiles in y
  if (g.M <= 64 || (small < big && fits)) return launch_linear_small(g, splits, st);
  return launch_linear_gemm(g, st);
}

int linear_check(int32_t T, int32_t K, int32_t N, int32_t act) {
  if (T < 0 || K < 1 || N < 1 || act < GROUTER_ACT_NONE || act > GROUTER_ACT_GELU) return GROUTER_ERR_INVALID_ARG;
  if (K % 8 || N % 8 || T > INT32_MAX - 256 || K > INT32_MAX - 256 || N > INT32_MAX - 256) return GROUTER_ERR_UNSUPPORTED;
  return GROUTER_OK;
}

}  // namespace
}  // namespace grouter

using namespace grouter;

extern "C" {

int grouter_linear_fwd(const void* x, const void* W, const void* bias, const void* residual, int32_t T, int32_t K, int32_t N, int32_t act, void* y,
                       void* pre, int32_t* status, void* stream) {
  if (const int e = linear_check(T, K, N, act)) return e;
  if (!W || !status || (T > 0 && (!x || !y))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(x, 16) || !aligned_to(W, 16) || !aligned_to(bias, 16) || !aligned_to(residual, 16) || !aligned_to(y, 16) || !aligned_to(pre, 16) ||
      !aligned_to(status, 4))
    return GROUTER_ERR_MISALIGNED;
  if (T == 0) return GROUTER_OK;
  LinearGemm g{};
  g.A = x; g.B = W; g.bias = bias; g.residual = residual; g.C = y; g.pre = pre;
  g.M = T; g.N = N; g.K = K; g.act = act; g.status = status;
  return launch_product(g, static_cast<cudaStream_t>(stream)) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

size_t grouter_linear_bwd_workspace_bytes(int32_t T, int32_t K, int32_t N, int32_t act) {
  if (linear_check(T, K, N, act) != GROUTER_OK) return 0;
  return linear_workspace(T, K, N, act).bytes;
}

int grouter_linear_bwd(const void* dy, const void* x, const void* W, const void* pre, int32_t T, int32_t K, int32_t N, int32_t act, void* dx,
                       void* dW, int32_t dW_dtype, float* db, void* workspace, int32_t* status, void* stream) {
  if (const int e = linear_check(T, K, N, act)) return e;
  if (!status || (!dx && !dW && !db) || (dW_dtype != GROUTER_BF16 && dW_dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  if (T > 0 && (!dy || !workspace || (dx && !W) || (dW && !x) || (act != GROUTER_ACT_NONE && !pre))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(dy, 16) || !aligned_to(x, 16) || !aligned_to(W, 16) || !aligned_to(pre, 16) || !aligned_to(dx, 16) || !aligned_to(dW, 16) ||
      !aligned_to(db, 4) || !aligned_to(workspace, 256) || !aligned_to(status, 4))
    return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {           // sums over no tokens
    if (dW && cudaMemsetAsync(dW, 0, (size_t)N * K * (dW_dtype == GROUTER_F32 ? 4 : 2), st) != cudaSuccess) return GROUTER_ERR_CUDA;
    if (db && cudaMemsetAsync(db, 0, (size_t)N * 4, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    return GROUTER_OK;
  }
  const LinearWorkspace w = linear_workspace(T, K, N, act);
  char* ws = static_cast<char*>(workspace);
  const void* dz = act == GROUTER_ACT_NONE ? dy : ws + w.dz;
  if (act != GROUTER_ACT_NONE || db) {
    const int rb = dz_row_blocks(T, N);
    // a single block of rows leaves the sums themselves
    float* partial = db ? (rb == 1 ? db : reinterpret_cast<float*>(ws + w.sums)) : nullptr;
    if (launch_dz(act, dy, pre, T, N, ws + w.dz, partial, rb, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    if (db && rb > 1 && launch_sum_rows(partial, rb, N, db, N, nullptr, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  }
  if (dx) {
    LinearGemm g{};
    g.A = dz; g.B = W; g.b_mn = 1; g.C = dx; g.M = T; g.N = K; g.K = N; g.act = GROUTER_ACT_NONE; g.status = status;
    if (launch_product(g, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  }
  if (dW) {
    const int pieces = dw_pieces(T, K, N);
    if (pieces == 1 && dW_dtype == GROUTER_BF16) {
      LinearGemm g{};
      g.A = dz; g.a_mn = 1; g.B = x; g.b_mn = 1; g.C = dW; g.M = N; g.N = K; g.K = T; g.act = GROUTER_ACT_NONE; g.status = status;
      if (launch_linear_gemm(g, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    } else {
      float* out = pieces == 1 ? static_cast<float*>(dW) : reinterpret_cast<float*>(ws + w.pieces);
      const int chunk = dw_chunk(T, pieces);
      if (launch_dense_gemm(dz, 1, x, 1, out, N, K, T, chunk, status, st) != cudaSuccess) return GROUTER_ERR_CUDA;
      if (pieces > 1) {
        const int64_t n4 = (int64_t)N * K / 4, want = (n4 + 255) / 256, cap = (int64_t)current_sms() * 8;
        const int grid = (int)(want < cap ? want : cap), real = cdiv(T, chunk);      // whole 64-token steps may leave the last piece out
        const cudaError_t e =
            dW_dtype == GROUTER_F32
                ? launch_dependent(sum_pieces_kernel<float>, dim3(grid), dim3(256), 0, st, out, real, n4, static_cast<float*>(dW))
                : launch_dependent(sum_pieces_kernel<__nv_bfloat16>, dim3(grid), dim3(256), 0, st, out, real, n4, static_cast<__nv_bfloat16*>(dW));
        if (e != cudaSuccess) return GROUTER_ERR_CUDA;
      }
    }
  }
  return GROUTER_OK;
}

}  // extern "C"
