// The products on 8-bit matrices for few tokens, where reading the weights once at HBM's pace is what counts.
//
//   LINEAR  C = x W^T + bias + residual        GLU  H = act(x Wg^T) (x Wu^T), as codes with a scale for 128 columns
//
// As for bf16 (linear_small.cu) the weight takes the M side of the tensor cores: a CTA multiplies 128 of its rows with a tile of TN tokens,
// the contraction cut over the S CTAs of a cluster, whose fp32 partial tiles are added up in rank order through shared memory
// (bit-reproducible).  GLU: 128 rows of both projections with an accumulator each, so that the 128 columns of a token's scale are in
// one place: a warp's lanes hold them, four each.
// A step is 128 deep, one block; its scales are bytes of 512-byte atoms that four steps share.  Every step brings the atoms along
// (3 % more bytes, from L2) and copies them into TMEM columns of its stage: the barriers that guard the stage guard them too.
//
// BF16 (up to 16 tokens): the tokens come as bf16, and four warps that have nothing else to do yet put each step's block into 8 bits on its
// way into the ring, so that no kernel has to run before this one (one token 4096 -> 1536: 4.4 us; from codes 3.9, and 1.9 for the kernel that makes them).
//
// Roles in a CTA as there: warp 0 loads, warp 1 issues, warps 2-5 bring the accumulators to shared memory, all eight share the epilogue.
// Every wait is bounded; on give-up the CTA raises STATUS_TIMEOUT, still meets the cluster's barriers, frees its TMEM and returns.
#include <cooperative_groups.h>

#include <type_traits>

#include "act.cuh"
#include "fp8.cuh"
#include "fp8_gemm.cuh"
#include "ptx.cuh"

namespace grouter {

namespace {

constexpr int FS_BM = 128, FS_BK = 128;
constexpr int FS_THREADS = 256;
constexpr int FS_MAX_SPLITS = 8;
constexpr int FS_PITCH = FS_BM + 4;                        // floats a row of the partial tile takes
__host__ __device__ constexpr int fs_stage_bytes(int tn, int tiles) { return (FS_BM * tiles + tn) * FS_BK + (tiles + 1) * FP8_ATOM; }
// as deep as two CTAs an SM allow (GLU: one)
__host__ __device__ constexpr int fs_stages(int tn, int tiles) {
  return tiles == 2 ? (tn == 16 ? 6 : tn == 128 ? 4 : 5) : (tn <= 32 ? 5 : tn == 64 ? 4 : 3);
}
__host__ __device__ constexpr int fs_smem(int tn, int tiles) { return fs_stages(tn, tiles) * fs_stage_bytes(tn, tiles) + 1024; }
// TMEM columns: the accumulators, then for every stage 4 of each weight tile's scales and 4 of the tokens'
__host__ __device__ constexpr int fs_tmem(int tn, int tiles) {
  const int need = tiles * tn + fs_stages(tn, tiles) * (tiles + 1) * 4;
  return need <= 64 ? 64 : need <= 128 ? 128 : need <= 256 ? 256 : 512;
}

struct Fp8SmallParams {
  int T, N, nk, across;          // tokens, outputs, 128-deep steps, scale atoms of a row
  const __nv_bfloat16* x;        // BF16: row t at x + t * ldx, K columns, 16-byte aligned rows
  int64_t ldx;
  int K;
  const __nv_bfloat16 *bias, *residual;
  __nv_bfloat16* out;            // LINEAR
  uint8_t *codes, *scales;       // GLU
  int act;
  int32_t* status;
  unsigned long long wait_limit_ns;
};

template <int TN, bool GLU, bool BF16>
__global__ void __launch_bounds__(FS_THREADS, GLU ? 1 : 2)
fp8_small_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmSW, const __grid_constant__ CUtensorMap tmW1,
                 const __grid_constant__ CUtensorMap tmSW1, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmSX,
                 const Fp8SmallParams p) {
  constexpr int TILES = GLU ? 2 : 1, STAGES = fs_stages(TN, TILES), STAGE_BYTES = fs_stage_bytes(TN, TILES), W_BYTES = FS_BM * FS_BK;
  constexpr int X_AT = TILES * W_BYTES, S_AT = X_AT + TN * FS_BK;        // places within a stage: weights, tokens, scales
  constexpr uint32_t TMEM_COLS = fs_tmem(TN, TILES), SCALES = TILES * TN;
  static_assert(STAGES * STAGE_BYTES >= TILES * TN * FS_PITCH * 4, "the partial tiles take the ring's place");
  // a stage is a multiple of 512 bytes, which its scales need, but not of the 1024 that a swizzled tile needs: operands of all stages
  // come first, then all scales
  constexpr int OPERANDS = S_AT;
  static_assert(OPERANDS % 1024 == 0, "stages on the swizzle's boundary");
  static_assert(!BF16 || TN == 16, "four warps of four tokens");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bars[2 * STAGES + 1];
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  namespace cg = cooperative_groups;
  cg::cluster_group cl = cg::this_cluster();
  const int S = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int n0 = blockIdx.x / S * FS_BM, t0 = blockIdx.y * TN;
  const int ks0 = (int)((int64_t)p.nk * rank / S), ks1 = (int)((int64_t)p.nk * (rank + 1) / S);
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t scale_base = smem_base + STAGES * OPERANDS;
  float* part = reinterpret_cast<float*>(smem_raw + (smem_base - ptx::smem_u32(smem_raw)));
  auto full_bar = [&](int s) { return ptx::smem_u32(&s_bars[s]); };
  auto empty_bar = [&](int s) { return ptx::smem_u32(&s_bars[STAGES + s]); };
  const uint32_t done_bar = ptx::smem_u32(&s_bars[2 * STAGES]);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < 2 * STAGES + 1; ++i) ptx::mbar_init(ptx::smem_u32(&s_bars[i]), BF16 && i < STAGES ? 5 : 1);      // full[]: the tokens' warps too
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmW);
    ptx::prefetch_tensormap(&tmSW);
    if (GLU) {
      ptx::prefetch_tensormap(&tmW1);
      ptx::prefetch_tensormap(&tmSW1);
    }
    if (!BF16) {
      ptx::prefetch_tensormap(&tmX);
      ptx::prefetch_tensormap(&tmSX);
    }
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(&s_tmem_base), TMEM_COLS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = s_tmem_base;
  volatile int* abort_flag = &s_abort;
  after_previous_kernel();           // set up while it was still ending; from here on its results are read
  let_next_kernel_start();

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      for (int ks = ks0; ks < ks1; ++ks) {
        if (!ptx::mbar_wait_bounded(empty_bar(s), ph ^ 1u, abort_flag, p.wait_limit_ns)) break;
        const uint32_t at = smem_base + s * OPERANDS, sc = scale_base + s * (TILES + 1) * FP8_ATOM, fb = full_bar(s);
        const int g = ks >> 2, atom = (n0 >> 7) * p.across + g;
        ptx::mbar_arrive_expect_tx(fb, (uint32_t)(BF16 ? STAGE_BYTES - TN * FS_BK - FP8_ATOM : STAGE_BYTES));
        ptx::tma_load_2d(at, &tmW, fb, ks * FS_BK, n0);                    // box {128 k, 128 rows}; what lies outside reads as zeros
        ptx::tma_load_2d(sc, &tmSW, fb, 0, atom);
        if (GLU) {
          ptx::tma_load_2d(at + W_BYTES, &tmW1, fb, ks * FS_BK, n0);
          ptx::tma_load_2d(sc + FP8_ATOM, &tmSW1, fb, 0, atom);
        }
        if (!BF16) {
          ptx::tma_load_2d(at + X_AT, &tmX, fb, ks * FS_BK, t0);           // box {128 k, TN tokens}
          ptx::tma_load_2d(sc + TILES * FP8_ATOM, &tmSX, fb, 0, (t0 >> 7) * p.across + g);
        }
        if (++s == STAGES) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    {
      const bool issues = ptx::elect_one();      // the warp stays together, one lane issues
      constexpr uint32_t idesc = ptx::make_idesc_fp8_scaled(FS_BM, TN);
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int ks = ks0; ks < ks1; ++ks) {
        if (!ptx::mbar_wait_bounded_warp(full_bar(s), ph, abort_flag, p.wait_limit_ns)) {
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t at = smem_base + s * OPERANDS, id = ptx::scale_byte(idesc, ks & 3);
        const uint64_t ds = ptx::make_smem_desc_scales(scale_base + s * (TILES + 1) * FP8_ATOM);
        const uint32_t t_s = tmem_base + SCALES + s * (TILES + 1) * 4;
        if (issues) {
#pragma unroll
          for (int i = 0; i <= TILES; ++i) ptx::tmem_copy_scales(t_s + 4 * i, ds + (i * FP8_ATOM >> 4));
#pragma unroll
          for (int kk = 0; kk < FS_BK / 32; ++kk) {
            const uint64_t dx = ptx::make_smem_desc_sw128(at + X_AT + kk * 32, 16, 1024);
#pragma unroll
            for (int i = 0; i < TILES; ++i)
              ptx::umma_fp8(tmem_base + i * TN, ptx::make_smem_desc_sw128(at + i * W_BYTES + kk * 32, 16, 1024), dx, id, t_s + 4 * i, t_s + 4 * TILES,
                            ks > ks0 || kk > 0 ? 1u : 0u);
          }
          ptx::umma_commit(empty_bar(s));
        }
        __syncwarp();
        if (++s == STAGES) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (ok && issues) ptx::umma_commit(done_bar);
    }
    __syncwarp();
  } else {
    // Eight lanes hold a token's block, each of four warps four tokens; the blocks of four steps are loaded and put into 8 bits side by side
    // and then go where their stages are free.  Columns of the tile whose tokens are not there keep what is in the stage: they are never read.
    if (BF16 && warp >= 4) {
      const int t = (warp - 4) * 4 + lane / Q_LANES, part_of = lane % Q_LANES;
      const bool any = (warp - 4) * 4 < p.T;             // of this warp's tokens
      const __nv_bfloat16* from = p.x + t * p.ldx + part_of * Q_LANE;
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int k0 = ks0; k0 < ks1 && ok; k0 += 4) {
        uint32_t w[4][8], e[4];
        if (any) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (k0 + i >= ks1) break;
            const int c = (k0 + i) * FS_BK;
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            const uint4 a = t < p.T && c + part_of * Q_LANE < p.K ? ld_stream16(from + c) : zero;
            const uint4 b = t < p.T && c + part_of * Q_LANE + 8 < p.K ? ld_stream16(from + c + 8) : zero;
            w[i][0] = a.x;
            w[i][1] = a.y;
            w[i][2] = a.z;
            w[i][3] = a.w;
            w[i][4] = b.x;
            w[i][5] = b.y;
            w[i][6] = b.z;
            w[i][7] = b.w;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (k0 + i >= ks1) break;
            bool inf;
            e[i] = block_exponent<__nv_bfloat16>(w[i], inf);
            const float2 inv = both(fp8_inverse(e[i]));
            const uint4 q = inf ? lane_codes<__nv_bfloat16, true>(w[i], inv) : lane_codes<__nv_bfloat16, false>(w[i], inv);
            w[i][0] = q.x;
            w[i][1] = q.y;
            w[i][2] = q.z;
            w[i][3] = q.w;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (k0 + i >= ks1) break;
          ok = ptx::mbar_wait_bounded_warp(empty_bar(s), ph ^ 1u, abort_flag, p.wait_limit_ns);
          if (!ok) break;
          if (t < p.T) {
            const uint32_t rows = smem_base + s * OPERANDS + X_AT, sc = scale_base + (s * (TILES + 1) + TILES) * FP8_ATOM;
            ptx::st_shared_v4(rows + t * FS_BK + ((part_of ^ (t & 7)) << 4), w[i][0], w[i][1], w[i][2], w[i][3]);       // 128-byte swizzle
            if (part_of == 0) ptx::st_shared_u8(sc + t * 16 + ((k0 + i) & 3), e[i]);
          }
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(full_bar(s));
          if (++s == STAGES) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
    }
    // the accumulators are complete: every load has landed and every MMA has read its stage, so the ring is free
    const int quad = warp & 3;                         // TMEM lane quadrant this warp may read
    if (warp < 6 && ptx::mbar_wait_bounded_warp(done_bar, 0u, abort_flag, p.wait_limit_ns)) {
      ptx::tc_fence_after();
      const int tv = min(TN, p.T - t0);
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int c = 0; c < TN; c += 16) {
          if (c < tv) {
            uint32_t r[16];
            ptx::tmem_ld16(tmem_base + ((uint32_t)(quad * 32) << 16) + i * TN + c, r);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 16; ++k) part[(i * TN + c + k) * FS_PITCH + quad * 32 + lane] = __uint_as_float(r[k]);
          }
        }
      }
    }
  }
  ptx::tc_fence_before();
  cl.sync();                                           // all partial tiles of the cluster are in place (or their CTAs gave up)
  const bool failed = *abort_flag != 0;
  const int tv = min(TN, p.T - t0), nv = min(FS_BM, p.N - n0);
  // A warp takes a token's 128 outputs, four a lane; the cluster's warps share the tokens.
  const int n = lane * 4;
  auto load4 = [&](const __nv_bfloat16* at, float (&f)[4]) {
    Pack<__nv_bfloat16, 4> q[1];
    *reinterpret_cast<uint2*>(&q[0]) = *reinterpret_cast<const uint2*>(at);
    const float2 a = pair_at(q, 0), b = pair_at(q, 1);
    f[0] = a.x;
    f[1] = a.y;
    f[2] = b.x;
    f[3] = b.y;
  };
  float bias[4] = {0.f, 0.f, 0.f, 0.f};
  if (!GLU && p.bias != nullptr && n < nv) load4(p.bias + n0 + n, bias);
  const int64_t pitch = GLU ? fp8_pitch(p.N) : 0, out_across = GLU ? fp8_atoms_across(p.N) : 0;
  const int step = S * (FS_THREADS / 32);
  // U tokens at a time, their sums over the CUTS partial tiles on their way together
  auto finish = [&](auto tokens, auto cuts, const float* const* parts) {
    constexpr int U = decltype(tokens)::value, CUTS = decltype(cuts)::value;
    for (int t = rank * (FS_THREADS / 32) + warp; t < tv; t += U * step) {
      float4 q[U][TILES][CUTS];
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int r = 0; r < CUTS; ++r)
            if (r < S && t + k * step < tv) q[k][i][r] = *reinterpret_cast<const float4*>(parts[r] + (i * TN + t + k * step) * FS_PITCH);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int tok = t + k * step;
        if (tok >= tv) break;
        float v[TILES][4];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          float4 a = q[k][i][0];
#pragma unroll
          for (int r = 1; r < CUTS; ++r) {
            if (r < S) {
              a.x += q[k][i][r].x;
              a.y += q[k][i][r].y;
              a.z += q[k][i][r].z;
              a.w += q[k][i][r].w;
            }
          }
          v[i][0] = a.x;
          v[i][1] = a.y;
          v[i][2] = a.z;
          v[i][3] = a.w;
        }
        if constexpr (!GLU) {
          if (n < nv) {                                // N is a multiple of 8: four outputs at a time are all there or none
            const int64_t at = (int64_t)(t0 + tok) * p.N + n0 + n;
            float res[4] = {0.f, 0.f, 0.f, 0.f};
            if (p.residual != nullptr) load4(p.residual + at, res);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[0][c] = v[0][c] + bias[c] + res[c];
            st_pack<__nv_bfloat16, 4>(p.out + at, v[0]);
          }
        } else {
          act_values(v[0], p.act);
          float top = 0.f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            v[0][c] = n < nv ? v[0][c] * v[TILES - 1][c] : 0.f;
            top = larger(top, v[0][c]);
          }
          top = lanes_top<32>(top);
          const bool inf = not_finite(top);
          if (inf) {
            top = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) top = larger_finite(top, v[0][c]);
            top = lanes_top<32>(top);
          }
          const uint32_t e = fp8_exponent(top);
          const float inv = fp8_inverse(e);
          if (n0 + n < pitch)
            *reinterpret_cast<uint32_t*>(p.codes + (t0 + tok) * pitch + n0 + n) = inf ? fp8_quad<true>(v[0], inv) : fp8_quad<false>(v[0], inv);
          if (lane == 0) p.scales[fp8_scale_at(t0 + tok, n0 >> 7, out_across)] = (uint8_t)e;
        }
      }
    }
  };
  if (S == 1) {                                        // this CTA's own tile: no way round over the cluster's addresses
    const float* own[1] = {part + n};
    finish(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{}, own);
  } else {
    const float* parts[FS_MAX_SPLITS];                 // the partial tiles in the cluster's shared memories
#pragma unroll
    for (int r = 0; r < FS_MAX_SPLITS; ++r) parts[r] = cl.map_shared_rank(part, r < S ? r : 0) + n;
    if (S <= 4) finish(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{}, parts);
    else finish(std::integral_constant<int, 1>{}, std::integral_constant<int, FS_MAX_SPLITS>{}, parts);
  }
  if (failed) {
    if (threadIdx.x == 0) atomicOr(p.status, STATUS_TIMEOUT);
    // give copies still in flight towards this CTA's shared memory time to land
    const uint64_t w0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - w0 < 2000000ull) __nanosleep(1000);
  }
  cl.sync();                                           // nobody leaves while its partial tile is read
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

template <int TN, bool GLU, bool BF16>
cudaError_t small_launch(const Fp8Gemm& g, int splits, cudaStream_t st) {
  constexpr int smem = fs_smem(TN, GLU ? 2 : 1);
  static bool configured[64] = {};       // the opt-in to more than 48 KB of dynamic shared memory, once per device
  auto kern = fp8_small_kernel<TN, GLU, BF16>;
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  CUtensorMap w, sw, w1, sw1, x, sx;
  bool ok = make_fp8_maps(&w, &sw, g.B, g.N, g.K, FS_BM);
  if (BF16) {
    x = w;
    sx = sw;
  } else {
    ok = ok && make_fp8_maps(&x, &sx, g.A, g.M, g.K, TN);
  }
  if (GLU) {
    ok = ok && make_fp8_maps(&w1, &sw1, g.B1, g.N, g.K, FS_BM);
  } else {
    w1 = w;
    sw1 = sw;
  }
  if (!ok) return cudaErrorInvalidValue;
  Fp8SmallParams p{};
  p.T = g.M;
  p.N = g.N;
  p.nk = (g.K + FS_BK - 1) / FS_BK;
  p.across = (int)fp8_atoms_across(g.K);
  p.x = static_cast<const __nv_bfloat16*>(g.x);
  p.ldx = g.ldx;
  p.K = g.K;
  p.bias = static_cast<const __nv_bfloat16*>(g.bias);
  p.residual = static_cast<const __nv_bfloat16*>(g.residual);
  p.out = GLU ? nullptr : static_cast<__nv_bfloat16*>(g.C);
  p.codes = GLU ? static_cast<uint8_t*>(g.C) : nullptr;
  p.scales = static_cast<uint8_t*>(g.out_scales);
  p.act = g.act;
  p.status = g.status;
  p.wait_limit_ns = DEFAULT_WAIT_LIMIT_NS;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((g.N + FS_BM - 1) / FS_BM * splits), (unsigned)((g.M + TN - 1) / TN));
  cfg.blockDim = dim3(FS_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = splits;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, w, sw, w1, sw1, x, sx, p);
}

template <bool GLU>
cudaError_t small_by_tokens(const Fp8Gemm& g, int splits, cudaStream_t st) {
  if (g.x) return g.M <= 16 ? small_launch<16, GLU, true>(g, splits, st) : cudaErrorInvalidValue;
  if (g.M <= 16) return small_launch<16, GLU, false>(g, splits, st);
  if (g.M <= 32) return small_launch<32, GLU, false>(g, splits, st);
  if (g.M <= 64) return small_launch<64, GLU, false>(g, splits, st);
  return small_launch<128, GLU, false>(g, splits, st);
}

}  // namespace

// Cuts of the contraction: as many as leave a CTA an SM of its own (4096 -> 4096: one token in 4 cuts, 128 CTAs, 5.1 us, in 8 cuts two to an
// SM 5.5; 128 tokens 8.1 and 11.2; 256 tokens 4096 -> 1536 in 4 cuts 7.9, in 8 10.1) and at least two 128-deep steps.  Clusters of
// eight do not find room everywhere: GLU, whose CTAs fill an SM, takes them up to three quarters of the SMs (16 tiles in eights 24.9 us,
// in fours 16.1).
int fp8_small_splits(int T, int N, int K, bool glu) {
  const int64_t tiles = (int64_t)((N + FS_BM - 1) / FS_BM) * ((T + 127) / 128);
  const int nk = (K + FS_BK - 1) / FS_BK, room = current_sms();
  int s = 1;
  while (s < FS_MAX_SPLITS && tiles * s * 2 <= (glu && s == 4 ? room * 3 / 4 : room) && nk >= 4 * s) s *= 2;
  return s;
}

cudaError_t launch_fp8_small(const Fp8Gemm& g, int splits, cudaStream_t st) {
  return g.B1.codes ? small_by_tokens<true>(g, splits, st) : small_by_tokens<false>(g, splits, st);
}

}  // namespace grouter
