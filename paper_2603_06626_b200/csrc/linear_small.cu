// The linear layer's product for few tokens:  C = act(B A^T + bias) + residual  with B [T, K] (the tokens), A a weight.
//
// With few tokens the 256 x 256 tiles of the CTA-pair core leave most SMs without work, and what counts is to read the weight once
// at HBM's pace from all of them.  Here the weight takes the M side of the tensor cores: a CTA multiplies 128 of its rows (outputs)
// with a tile of TN tokens (16, 32, 64 or 128), accumulator [128 outputs, TN tokens] in TMEM, and the contraction is cut over the S
// CTAs of a cluster (S = 1, 2, 4, 8), so that e.g. one token through a 4096 x 4096 weight keeps 256 CTAs loading, two to an SM, some
// 90 KB of the weight on its way into each.  The CTAs then leave their fp32 partial tiles in shared memory, every one adds up
// a share of the outputs over the S tiles in rank order (bit-reproducible), applies bias, activation and residual and writes.
//
// Bound by latency more than by the weight's bytes.  Measured, weight 4096 x 4096 (33.5 MB, 5.2 us at a plain copy's pace): one token
// 9.9 us with ten weights in turn (335 MB, from HBM), 8.5 with three (100 MB, which stay in L2); with three, 64 tokens 12 us and 256
// tokens 18; 128 x 128 with one token 4.1 us, which is what launch, set-up and the cluster's two barriers take.  A CTA has eight steps
// and a ring of six, so its first load and its epilogue are most of its time.
//
// GATED: the up-projection of the gated feed-forward block, H = act(x Wg^T) * (x Wu^T).  A CTA's 128 weight rows are 64 of the gate and the
// 64 of the other projection that belong to them, so it has both accumulators of an output in its partial tile.
//
// Roles in a CTA: warp 0 loads (TMA, ring of STAGES 64-deep steps), warp 1 issues the MMAs, warps 2-5 bring the accumulator to
// shared memory; all six share the epilogue.  Every wait is bounded, as in the CTA-pair core: on give-up the CTA raises
// STATUS_TIMEOUT, still meets the cluster's barriers, frees its TMEM and returns.
#include <cooperative_groups.h>

#include "act.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace grouter {

constexpr int LS_BM = 128, LS_BK = 64;
constexpr int LS_THREADS = 192;
constexpr int LS_MAX_SPLITS = 8;
constexpr int LS_PITCH = LS_BM + 4;                        // floats a row of the partial tile takes
__host__ __device__ constexpr int ls_stage_bytes(int tn) { return (LS_BM + tn) * LS_BK * 2; }
// as deep as two CTAs an SM allow
__host__ __device__ constexpr int ls_stages(int tn) { return tn == 16 ? 6 : tn == 32 ? 5 : tn == 64 ? 4 : 3; }
__host__ __device__ constexpr int ls_smem(int tn) { return ls_stages(tn) * ls_stage_bytes(tn) + 1024; }

struct LinearSmallParams {
  int T, N, nk;                  // tokens, outputs, 64-deep steps of the contraction
  const __nv_bfloat16 *bias, *residual;
  __nv_bfloat16 *out, *pre;
  int act;
  int32_t* status;
  unsigned long long wait_limit_ns;
};

template <int TN, bool A_MN, bool GATED>
__global__ void __launch_bounds__(LS_THREADS, 2) linear_small_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                                                                     const LinearSmallParams p) {
  constexpr int STAGES = ls_stages(TN), STAGE_BYTES = ls_stage_bytes(TN), A_BYTES = LS_BM * LS_BK * 2;
  constexpr uint32_t TMEM_COLS = TN < 32 ? 32 : TN;
  static_assert(STAGES * STAGE_BYTES >= TN * LS_PITCH * 4, "the partial tile takes the ring's place");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bars[2 * STAGES + 1];
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  namespace cg = cooperative_groups;
  cg::cluster_group cl = cg::this_cluster();
  const int S = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int tile = blockIdx.x / S;
  constexpr int OUT = GATED ? LS_BM / 2 : LS_BM;      // outputs of a CTA
  const int n0 = tile * OUT, t0 = blockIdx.y * TN;
  const int ks0 = (int)((int64_t)p.nk * rank / S), ks1 = (int)((int64_t)p.nk * (rank + 1) / S);
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  float* part = reinterpret_cast<float*>(smem_raw + (smem_base - ptx::smem_u32(smem_raw)));
  auto full_bar = [&](int s) { return ptx::smem_u32(&s_bars[s]); };
  auto empty_bar = [&](int s) { return ptx::smem_u32(&s_bars[STAGES + s]); };
  const uint32_t done_bar = ptx::smem_u32(&s_bars[2 * STAGES]);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < 2 * STAGES + 1; ++i) ptx::mbar_init(ptx::smem_u32(&s_bars[i]), 1);
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmA);
    ptx::prefetch_tensormap(&tmB);
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
        const uint32_t sa = smem_base + s * STAGE_BYTES, sb = sa + A_BYTES;
        ptx::mbar_arrive_expect_tx(full_bar(s), (uint32_t)STAGE_BYTES);
        if (GATED) {
          ptx::tma_load_2d(sa, &tmA, full_bar(s), ks * LS_BK, n0);             // 2 x box {64 k, 64 rows}; rows beyond the last read as zeros
          ptx::tma_load_2d(sa + A_BYTES / 2, &tmA, full_bar(s), ks * LS_BK, p.N + n0);
        } else if (!A_MN) {
          ptx::tma_load_2d(sa, &tmA, full_bar(s), ks * LS_BK, n0);             // box {64 k, 128 rows}; rows beyond N read as zeros
        } else {
          ptx::tma_load_2d(sa, &tmA, full_bar(s), n0, ks * LS_BK);             // 2 x box {64 rows, 64 k}
          ptx::tma_load_2d(sa + A_BYTES / 2, &tmA, full_bar(s), n0 + 64, ks * LS_BK);
        }
        ptx::tma_load_2d(sb, &tmB, full_bar(s), ks * LS_BK, t0);               // box {64 k, TN tokens}; tokens beyond T read as zeros
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
      constexpr uint32_t idesc = ptx::make_idesc_bf16(LS_BM, TN, A_MN, false);
      // operand layouts as in the CTA-pair core (gemm.cu)
      constexpr uint32_t a_lbo = A_MN ? A_BYTES / 2 : 16, a_kadv = A_MN ? 2048 : 32;
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int ks = ks0; ks < ks1; ++ks) {
        if (!ptx::mbar_wait_bounded_warp(full_bar(s), ph, abort_flag, p.wait_limit_ns)) {
          ok = false;
          break;
        }
        ptx::tc_fence_after();
        const uint32_t sa = smem_base + s * STAGE_BYTES, sb = sa + A_BYTES;
        if (issues) {
#pragma unroll
          for (int kk = 0; kk < LS_BK / 16; ++kk) {
            const uint64_t da = ptx::make_smem_desc_sw128(sa + kk * a_kadv, a_lbo, 1024);
            const uint64_t db = ptx::make_smem_desc_sw128(sb + kk * 32, 16, 1024);
            ptx::umma_bf16(tmem_base, da, db, idesc, ks > ks0 || kk > 0 ? 1u : 0u);
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
    // the accumulator is complete: every load has landed and every MMA has read its stage, so the ring is free
    const int quad = warp & 3;                         // TMEM lane quadrant this warp may read
    if (ptx::mbar_wait_bounded_warp(done_bar, 0u, abort_flag, p.wait_limit_ns)) {
      ptx::tc_fence_after();
      const int tv = min(TN, p.T - t0);
#pragma unroll
      for (int c = 0; c < TN; c += 16) {
        if (c < tv) {
          uint32_t r[16];
          ptx::tmem_ld16(tmem_base + ((uint32_t)(quad * 32) << 16) + c, r);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) part[(c + i) * LS_PITCH + quad * 32 + lane] = __uint_as_float(r[i]);
        }
      }
    }
  }
  ptx::tc_fence_before();
  cl.sync();                                           // all partial tiles of the cluster are in place (or their CTAs gave up)
  const bool failed = *abort_flag != 0;
  const int tv = min(TN, p.T - t0), nv = min(OUT, p.N - n0);
  auto load4 = [&](const __nv_bfloat16* q, float (&f)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(q);
    const float2 lo = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
    const float2 hi = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
    f[0] = lo.x;
    f[1] = lo.y;
    f[2] = hi.x;
    f[3] = hi.y;
  };
  auto store4 = [&](__nv_bfloat16* q, const float (&f)[4]) {
    uint2 u;
    *reinterpret_cast<__nv_bfloat162*>(&u.x) = __floats2bfloat162_rn(f[0], f[1]);
    *reinterpret_cast<__nv_bfloat162*>(&u.y) = __floats2bfloat162_rn(f[2], f[3]);
    *reinterpret_cast<uint2*>(q) = u;
  };
  // A thread keeps its four outputs n .. n + 3 and goes down the tokens, a whole cluster's threads sharing them.
  static_assert(LS_THREADS % (OUT / 4) == 0, "a thread's outputs stay the same from step to step");
  const int n = (threadIdx.x % (OUT / 4)) * 4, per_step = LS_THREADS / (OUT / 4);
  if (GATED && n < nv) {
    const float* parts[LS_MAX_SPLITS];
#pragma unroll
    for (int r = 0; r < LS_MAX_SPLITS; ++r) parts[r] = cl.map_shared_rank(part, r < S ? r : 0) + n;
    for (int t = rank * per_step + threadIdx.x / (OUT / 4); t < tv; t += S * per_step) {
      float4 q[LS_MAX_SPLITS][2];
#pragma unroll
      for (int r = 0; r < LS_MAX_SPLITS; ++r) {
        if (r < S) {
          q[r][0] = *reinterpret_cast<const float4*>(parts[r] + t * LS_PITCH);
          q[r][1] = *reinterpret_cast<const float4*>(parts[r] + t * LS_PITCH + OUT);
        }
      }
      float g[4] = {q[0][0].x, q[0][0].y, q[0][0].z, q[0][0].w}, u[4] = {q[0][1].x, q[0][1].y, q[0][1].z, q[0][1].w};
#pragma unroll
      for (int r = 1; r < LS_MAX_SPLITS; ++r) {
        if (r < S) {
          g[0] += q[r][0].x;
          g[1] += q[r][0].y;
          g[2] += q[r][0].z;
          g[3] += q[r][0].w;
          u[0] += q[r][1].x;
          u[1] += q[r][1].y;
          u[2] += q[r][1].z;
          u[3] += q[r][1].w;
        }
      }
      if (p.pre) {
        __nv_bfloat16* to = p.pre + (int64_t)(t0 + t) * 2 * p.N + n0 + n;
        store4(to, g);
        store4(to + p.N, u);
      }
      act_values(g, p.act);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] *= u[i];
      store4(p.out + (int64_t)(t0 + t) * p.N + n0 + n, g);
    }
  } else if (n < nv) {                                        // N is a multiple of 8: four outputs at a time are all there or none
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.bias) load4(p.bias + n0 + n, bias);
    auto finish = [&](int t, float4 a) {
      float v[4] = {a.x + bias[0], a.y + bias[1], a.z + bias[2], a.w + bias[3]};
      const int64_t at = (int64_t)(t0 + t) * p.N + n0 + n;
      float res[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.residual) load4(p.residual + at, res);
      if (p.pre) store4(p.pre + at, v);
      if (p.act == GROUTER_ACT_RELU) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = act_value<GROUTER_ACT_RELU>(v[q]);
      } else if (p.act == GROUTER_ACT_SILU) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = act_value<GROUTER_ACT_SILU>(v[q]);
      } else if (p.act == GROUTER_ACT_GELU) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = act_value<GROUTER_ACT_GELU>(v[q]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += res[q];
      store4(p.out + at, v);
    };
    const int first = rank * per_step + threadIdx.x / (LS_BM / 4);
    if (S == 1) {                                      // this CTA's own tile: no way round over the cluster's addresses
#pragma unroll 4
      for (int t = first; t < tv; t += per_step) finish(t, *reinterpret_cast<const float4*>(part + t * LS_PITCH + n));
    } else {
      const float* parts[LS_MAX_SPLITS];               // the partial tiles in the cluster's shared memories
#pragma unroll
      for (int r = 0; r < LS_MAX_SPLITS; ++r) parts[r] = cl.map_shared_rank(part, r < S ? r : 0) + n;
      for (int t = first; t < tv; t += S * per_step) {
        float4 q[LS_MAX_SPLITS];
#pragma unroll
        for (int r = 0; r < LS_MAX_SPLITS; ++r)
          if (r < S) q[r] = *reinterpret_cast<const float4*>(parts[r] + t * LS_PITCH);
        float4 a = q[0];
#pragma unroll
        for (int r = 1; r < LS_MAX_SPLITS; ++r) {
          if (r < S) {
            a.x += q[r].x;
            a.y += q[r].y;
            a.z += q[r].z;
            a.w += q[r].w;
          }
        }
        finish(t, a);
      }
    }
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

namespace {

template <int TN, bool A_MN, bool GATED>
cudaError_t small_launch(const LinearGemm& g, int splits, cudaStream_t st) {
  static bool configured[64] = {};       // the opt-in to more than 48 KB of dynamic shared memory, once per device
  auto kern = linear_small_kernel<TN, A_MN, GATED>;
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, ls_smem(TN));
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  // here the weight is the M side: g.B of the product as the other kernel sees it
  CUtensorMap a, b;
  const bool ok = (GATED  ? make_bf16_tile_map(&a, g.B, 2 * (uint64_t)g.N, g.K, LS_BM / 2)
                   : A_MN ? make_bf16_tile_map(&a, g.B, g.K, g.N, 64)
                          : make_bf16_tile_map(&a, g.B, g.N, g.K, LS_BM)) &&
                  make_bf16_tile_map(&b, g.A, g.M, g.K, TN);
  if (!ok) return cudaErrorInvalidValue;
  LinearSmallParams p{};
  p.T = g.M;
  p.N = g.N;
  p.nk = (g.K + LS_BK - 1) / LS_BK;
  p.bias = static_cast<const __nv_bfloat16*>(g.bias);
  p.residual = static_cast<const __nv_bfloat16*>(g.residual);
  p.out = static_cast<__nv_bfloat16*>(g.C);
  p.pre = static_cast<__nv_bfloat16*>(g.pre);
  p.act = g.act;
  p.status = g.status;
  p.wait_limit_ns = DEFAULT_WAIT_LIMIT_NS;
  cudaLaunchConfig_t cfg{};
  constexpr int OUT = GATED ? LS_BM / 2 : LS_BM;
  cfg.gridDim = dim3((unsigned)((g.N + OUT - 1) / OUT * splits), (unsigned)((g.M + TN - 1) / TN));
  cfg.blockDim = dim3(LS_THREADS);
  cfg.dynamicSmemBytes = ls_smem(TN);
  cfg.stream = st;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = splits;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, a, b, p);
}

template <bool A_MN, bool GATED>
cudaError_t small_by_tokens(const LinearGemm& g, int splits, cudaStream_t st) {
  if (g.M <= 16) return small_launch<16, A_MN, GATED>(g, splits, st);
  if (g.M <= 32) return small_launch<32, A_MN, GATED>(g, splits, st);
  if (g.M <= 64) return small_launch<64, A_MN, GATED>(g, splits, st);
  return small_launch<128, A_MN, GATED>(g, splits, st);
}

}  // namespace

// Cuts of the contraction: as many as fit two CTAs an SM at once, and no CTA left with fewer than four 64-deep steps.
int linear_small_splits(int T, int N, int K) {
  const int64_t tiles = (int64_t)((N + LS_BM - 1) / LS_BM) * ((T + 127) / 128);
  const int nk = (K + LS_BK - 1) / LS_BK, room = 2 * current_sms();
  int s = 1;
  while (s < LS_MAX_SPLITS && tiles * s * 2 <= room && nk >= 8 * s) s *= 2;
  return s;
}

cudaError_t launch_linear_small(const LinearGemm& g, int splits, cudaStream_t st) {
  return g.b_mn ? small_by_tokens<true, false>(g, splits, st) : small_by_tokens<false, false>(g, splits, st);
}

// As linear_small_splits, but one CTA an SM, which streams twice as long (24 tiles of 64 tokens, 4096 deep: in 4 cuts 11.7 us, in 8 13.0; 128 tokens
// 14.0 and 17.5; one token 8.9 and 8.4), unless that leaves a CTA 64 steps or more (d 8192, hidden 4096, both products: 128 tokens in 2 cuts 55
// us, in 4 48; hidden 8192 in 1 cut 93, in 2 79; one token 69 and 66; 2048 deep, 128 tiles, 8 tokens in 1 cut 23.2, in 2 24.3).
int gated_small_splits(int T, int H, int K) {
  const int64_t tiles = (int64_t)((2 * (int64_t)H + LS_BM - 1) / LS_BM) * ((T + 127) / 128);
  const int nk = (K + LS_BK - 1) / LS_BK, sms = current_sms();
  int s = 1;
  while (s < LS_MAX_SPLITS && tiles * s * 2 <= (nk >= 64 * s ? 2 * sms : sms) && nk >= 8 * s) s *= 2;
  return s;
}

cudaError_t launch_gated_small(const GatedGemm& g, int splits, cudaStream_t st) {
  LinearGemm l{};
  l.A = g.A; l.B = g.W; l.C = g.h; l.pre = g.pre; l.M = g.T; l.N = g.H; l.K = g.K; l.act = g.act; l.status = g.status;
  return small_by_tokens<false, true>(l, splits, st);
}

}  // namespace grouter
