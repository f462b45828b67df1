// Products of matrices in 8 bits (fp8.cuh) on the sm_100a tensor cores, scales applied on the way.
//
//   LINEAR  C = A B^T + bias + residual        C_mn = sum_b 2^(ea(m,b) + eb(n,b)) sum_{k in block b} ca_mk cb_nk, bf16 or f32 out
//   GLU     [G|U] = A [Wg;Wu]^T,  H = act(G) U, out as codes with a scale for 128 columns: the next product's operand
//   TWO     two LINEAR products in one launch: the backward pass of the linear layer
//
// The CTA-pair pipeline of the bf16 products (gemm.cu): tiles of 256 x 256, five 32 KB stages in each CTA, here 128 deep; warp 0
// loads, warp 1 of the leader issues, warps 2-9 empty the accumulator.  A block of 128 is exactly one step, so its scale is one byte a
// row, and four steps' bytes are the 512-byte atom that lies in memory: every fourth step brings one atom of A's rows and the two of
// all 256 of B's rows (both CTAs multiply with all of B) into shared memory and from there into TMEM.
// TMEM: two accumulators of 256 columns would be all of it.  They overlap by the 32 columns that two sets of scales need: accumulator
// 1 starts at column 224.  Whoever reads the shared columns of a tile reads them first and says so (`over`), and the next tile's
// products wait for that, while its operands arrive.
// Every wait is bounded, as in gemm.cu.
//
// Measured: 8192 x 4096 x 4096 95-107 us, 8192^3 381-445 (2.5 to 2.9 PFLOP/s by the clock that the power limit leaves); GLU 16384 tokens, 4096 ->
// 1536 126 us with the tensor pipe 80 % active; 16384 x 1536 x 4096 with a residual 85-100 (119 in a loop at the power
// limit), 57 %: every 12 steps a tile of 128 KB goes out and one of the residual comes in.  A step takes its 32 KB per SM in 256 tensor
// cycles, twice the pace at which bf16 tiles need theirs, so tiles smaller than 256 x 256 are out.
#include "act.cuh"
#include "fp8.cuh"
#include "fp8_gemm.cuh"
#include "ptx.cuh"

namespace grouter {

namespace {

constexpr int F8_BM = 128, F8_PM = 256, F8_BN = 256, F8_BNH = 128, F8_BK = 128;
constexpr int F8_STAGES = 5;
constexpr int F8_A_BYTES = F8_BM * F8_BK, F8_B_BYTES = F8_BNH * F8_BK;       // 16 KB each
constexpr int F8_STAGE_BYTES = F8_A_BYTES + F8_B_BYTES;
constexpr int F8_SCALE_BYTES = 3 * FP8_ATOM;          // A's rows of this CTA, B's first and second 128 rows
constexpr int F8_EPI_WARPS = 8;
constexpr int F8_THREADS = 64 + 32 * F8_EPI_WARPS;
constexpr int F8_BLOCK_BYTES = 32 * 64;               // one staging block: 32 rows x 64 bytes
constexpr int F8_EPI_BLOCKS = 3;
constexpr int F8_STAGING = F8_EPI_WARPS * F8_EPI_BLOCKS * F8_BLOCK_BYTES;
constexpr int F8_SMEM = F8_STAGES * (F8_STAGE_BYTES + F8_SCALE_BYTES) + F8_STAGING + 1024 /*align*/ + 256 /*barriers*/;
constexpr uint32_t F8_ACC1 = 224, F8_SCALES = 480, F8_SCALE_SET = 16;       // TMEM columns: accumulator 1, the two sets of scales (A +0, B +8)
constexpr int F8_RASTER = 8;

enum F8Mode { F8_LINEAR = 0, F8_GLU = 1, F8_TWO = 2 };      // TWO: two LINEAR products in one launch

struct F8Product {
  int M, N, K;                   // GLU: N = hidden columns
  int tiles_m, tiles_n, across;  // across: scale atoms of a row of 128s
  int pieces, piece_steps;       // f32 out: the contraction cut into pieces of so many steps, a multiple of four, each with a matrix of its own
  int piece_rows;                // ... of so many rows, M rounded up to whole staging blocks
  int tiles;                     // of all pieces
  const __nv_bfloat16 *bias, *residual;
  int out_f32;
};
struct F8Maps {
  CUtensorMap A, SA, B, SB, C;
};
struct F8Params {
  F8Maps maps[2];                // GLU: B and SB of the second are the other projection
  F8Product of[2];
  int ahead;                     // TWO: tiles of the second product that a pair has time for while others have one more of the first
  int act;
  uint8_t* out_scales;           // GLU
  int32_t* status;
  unsigned long long wait_limit_ns;
  int waits_at_end;              // as in gemm.cu
};

// The i-th tile of a pair; false behind its last.  TWO: the first product's tiles go round the pairs; the second's, whose contraction is shorter,
// first to those pairs that the last round leaves without a tile, `ahead` each, then round all of them.
template <int MODE>
__device__ __forceinline__ bool f8_pick(const F8Params& p, int i, int pair, int n_pairs, int& which, int& t) {
  which = 0;
  t = pair + i * n_pairs;
  if (MODE != F8_TWO) return t < p.of[0].tiles;
  if (t < p.of[0].tiles) return true;
  which = 1;
  const int late = p.of[0].tiles % n_pairs;          // pairs with one more
  int r = i - p.of[0].tiles / n_pairs - (pair < late ? 1 : 0);
  if (late > 0) {
    if (pair >= late && r < p.ahead) {
      t = r * (n_pairs - late) + pair - late;
      return t < p.of[1].tiles;
    }
    t = p.ahead * (n_pairs - late);
    if (pair >= late) r -= p.ahead;
  } else {
    t = 0;
  }
  t += r * n_pairs + pair;
  return t < p.of[1].tiles;
}

struct F8Tile {
  int row0, col0, m_valid, n_valid;
  int step0, steps, out_row;     // first step, steps; row of the output's first row of the piece
};

template <int MODE>
__device__ __forceinline__ F8Tile f8_tile(const F8Product& p, int t, int rank) {
  // bands of tile rows, down the band first, as for the bf16 products: the pairs in flight share rows of A and columns of B
  const int per = p.tiles_m * p.tiles_n, piece = MODE == F8_GLU ? 0 : t / per;
  t -= piece * per;
  const int band = t / (F8_RASTER * p.tiles_n), in_band = t - band * F8_RASTER * p.tiles_n;
  const int rows = min(F8_RASTER, p.tiles_m - band * F8_RASTER);
  const int nt = in_band / rows, mt = band * F8_RASTER + (in_band - nt * rows);
  constexpr int cols = MODE == F8_GLU ? F8_BNH : F8_BN;
  F8Tile ti;
  ti.row0 = mt * F8_PM + rank * F8_BM;
  ti.col0 = nt * cols;
  ti.m_valid = min(F8_BM, p.M - ti.row0);
  ti.n_valid = min(cols, p.N - ti.col0);
  ti.step0 = piece * p.piece_steps;
  ti.steps = min(p.piece_steps, (p.K + F8_BK - 1) / F8_BK - ti.step0);
  ti.out_row = piece * p.piece_rows;
  return ti;
}

template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(F8_THREADS, 1) fp8_gemm_kernel(const __grid_constant__ F8Params p) {
  extern __shared__ uint8_t smem_raw[];
  // the same offsets in both CTAs of the pair: descriptors and multicast commits name both
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t staging = smem_base + F8_STAGES * F8_STAGE_BYTES;
  const uint32_t scale_base = staging + F8_STAGING;
  const uint32_t bar_base = scale_base + F8_STAGES * F8_SCALE_BYTES;
  //   full[s] leader only, one arrival with the bytes of both CTAs      empty[s] each CTA, by the leader's commit
  //   tmem_full[a] each CTA, by the leader's commit                      tmem_empty[a] leader only, one arrival an epilogue warp
  //   over: leader only, one arrival of the eight warps that read the columns which both accumulators have
  //   scales[b]: leader only, the products that read set b are done      top[quad]: GLU, the two warps that share rows have their maxima in place
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (F8_STAGES + s); };
  auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * F8_STAGES + a); };
  auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * F8_STAGES + 2 + a); };
  const uint32_t over_bar = bar_base + 8u * (2 * F8_STAGES + 4);
  auto scales_bar = [&](int b) { return bar_base + 8u * (2 * F8_STAGES + 5 + b); };
  auto top_bar = [&](int q) { return bar_base + 8u * (2 * F8_STAGES + 7 + q); };
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  __shared__ float s_top[MODE == F8_GLU ? 2 : 1][2][F8_BM];         // [tile parity][half of the columns][row]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)ptx::cluster_ctarank();
  const int pair_id = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < F8_STAGES; ++s) {
      ptx::mbar_init(full_bar(s), 1);
      ptx::mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(tfull_bar(a), 1);
      ptx::mbar_init(tempty_bar(a), 2 * F8_EPI_WARPS);
      ptx::mbar_init(scales_bar(a), 1);
    }
    ptx::mbar_init(over_bar, F8_EPI_WARPS);
    for (int q = 0; q < 4; ++q) ptx::mbar_init(top_bar(q), 2);
    ptx::fence_mbar_init();
    for (int i = 0; i < (MODE == F8_TWO ? 2 : 1); ++i) {
      const F8Maps& m = p.maps[i];
      for (const CUtensorMap* map : {&m.A, &m.SA, &m.B, &m.SB, &m.C}) ptx::prefetch_tensormap(map);
    }
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(ptx::smem_u32(&s_tmem_base), 512);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync_all();      // the peer's barriers are initialised and its TMEM is allocated
  ptx::tc_fence_after();
  const uint32_t tmem_base = s_tmem_base;
  volatile int* abort_flag = &s_abort;
  if (!p.waits_at_end) after_previous_kernel();      // set up while the kernel before was still ending; from here on its results are read
  let_next_kernel_start();

  if (warp == 0) {
    // ===================== TMA producer (both CTAs) =====================
    if (lane == 0) {
      const uint64_t keep_a = ptx::l2_policy_evict_normal(), keep_b = ptx::l2_policy_evict_last();
      int s = 0;
      uint32_t ph = 0;
      int which, t;
      for (int i = 0; f8_pick<MODE>(p, i, pair_id, n_pairs, which, t) && !*abort_flag; ++i) {
        const F8Tile ti = f8_tile<MODE>(p.of[which], t, rank);
        const F8Maps& m = p.maps[which];
        const int across = p.of[which].across;
        const CUtensorMap* b_map = MODE == F8_GLU && rank == 1 ? &p.maps[1].B : &m.B;
        const int b_row = MODE == F8_GLU ? ti.col0 : ti.col0 + rank * F8_BNH;
        const int sa_atom = (ti.row0 >> 7) * across, sb_atom = (ti.col0 >> 7) * across;
        bool ok = true;
        for (int ks = 0; ks < ti.steps; ++ks) {
          if (!ptx::mbar_wait_bounded(empty_bar(s), ph ^ 1u, abort_flag, p.wait_limit_ns)) {
            ok = false;
            break;
          }
          const bool scales = (ks & 3) == 0;
          const uint32_t sa = smem_base + s * F8_STAGE_BYTES, sb = sa + F8_A_BYTES, sc = scale_base + s * F8_SCALE_BYTES;
          if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(s), 2 * (F8_STAGE_BYTES + (scales ? F8_SCALE_BYTES : 0)));
          const uint32_t fb = ptx::map_to_cta(full_bar(s), 0);      // both CTAs' bytes complete on the leader's barrier
          if (scales) {
            const int g = (ti.step0 + ks) >> 2;
            ptx::tma_load_2d_pair(sc, &m.SA, fb, 0, sa_atom + g, keep_a);
            ptx::tma_load_2d_pair(sc + FP8_ATOM, &m.SB, fb, 0, sb_atom + g, keep_b);
            if (MODE == F8_GLU) ptx::tma_load_2d_pair(sc + 2 * FP8_ATOM, &p.maps[1].SB, fb, 0, sb_atom + g, keep_b);
            else ptx::tma_load_2d_pair(sc + 2 * FP8_ATOM, &m.SB, fb, 0, sb_atom + across + g, keep_b);      // beyond the last row: zeros
          }
          ptx::tma_load_2d_pair(sa, &m.A, fb, (ti.step0 + ks) * F8_BK, ti.row0, keep_a);      // box {128 k, 128 rows}
          ptx::tma_load_2d_pair(sb, b_map, fb, (ti.step0 + ks) * F8_BK, b_row, keep_b);
          if (++s == F8_STAGES) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (!ok) break;
      }
      // every stage release the leader has multicast to this CTA must have landed before the CTA may exit
      for (int i = 0; i < F8_STAGES && !*abort_flag; ++i) {
        if (!ptx::mbar_wait_bounded(empty_bar(s), ph ^ 1u, abort_flag, p.wait_limit_ns)) break;
        if (++s == F8_STAGES) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ===================== MMA issuer (leader CTA only): the warp together, one lane issues =====================
    if (rank == 0) {
      const bool issues = ptx::elect_one();
      constexpr uint32_t idesc = ptx::make_idesc_fp8_scaled(F8_PM, F8_BN);
      constexpr uint16_t both = 3, leader = 1;
      const uint64_t da0 = ptx::make_smem_desc_sw128(smem_base, 16, 1024), db0 = ptx::make_smem_desc_sw128(smem_base + F8_A_BYTES, 16, 1024);
      const uint32_t a_hi = (uint32_t)(da0 >> 32), b_hi = (uint32_t)(db0 >> 32);
      int s = 0, acc = 0, set = 0;
      uint32_t ph = 0, acc_ph = 0, over_ph = 0, set_ph = 0;
      bool first = true;
      int which, t;
      for (int i = 0; f8_pick<MODE>(p, i, pair_id, n_pairs, which, t) && !__any_sync(0xffffffffu, *abort_flag); ++i) {
        if (!ptx::mbar_wait_bounded_warp(tempty_bar(acc), acc_ph ^ 1u, abort_flag, p.wait_limit_ns)) break;
        if (!first) {
          if (!ptx::mbar_wait_bounded_warp(over_bar, over_ph, abort_flag, p.wait_limit_ns)) break;
          over_ph ^= 1u;
        }
        first = false;
        ptx::tc_fence_after();
        const uint32_t d_tmem = tmem_base + (acc ? F8_ACC1 : 0u);
        const int steps = f8_tile<MODE>(p.of[which], t, 0).steps;
        bool ok = true;
        for (int ks = 0; ks < steps; ++ks) {
          if (!ptx::mbar_wait_bounded_warp(full_bar(s), ph, abort_flag, p.wait_limit_ns)) {
            ok = false;
            break;
          }
          const uint32_t t_sa = tmem_base + F8_SCALES + set * F8_SCALE_SET, t_sb = t_sa + 8;
          if ((ks & 3) == 0) {
            if (!ptx::mbar_wait_bounded_warp(scales_bar(set), set_ph ^ 1u, abort_flag, p.wait_limit_ns)) {
              ok = false;
              break;
            }
            ptx::tc_fence_after();
            const uint64_t ds = ptx::make_smem_desc_scales(scale_base + s * F8_SCALE_BYTES);
            if (issues) {
              ptx::tmem_copy_scales_pair(t_sa, ds);
              ptx::tmem_copy_scales_pair(t_sb, ds + (FP8_ATOM >> 4));
              ptx::tmem_copy_scales_pair(t_sb + 4, ds + (2 * FP8_ATOM >> 4));
            }
            __syncwarp();
          }
          const uint32_t a_lo = (uint32_t)da0 + s * (F8_STAGE_BYTES >> 4), b_lo = (uint32_t)db0 + s * (F8_STAGE_BYTES >> 4);
          const uint32_t id = ptx::scale_byte(idesc, ks & 3);
          const bool last_of_set = (ks & 3) == 3 || ks == steps - 1;
          if (issues) {
#pragma unroll
            for (int kk = 0; kk < F8_BK / 32; ++kk)
              ptx::umma_fp8_pair(d_tmem, a_lo + kk * 2, a_hi, b_lo + kk * 2, b_hi, id, t_sa, t_sb, (ks | kk) != 0 ? 1u : 0u);
            ptx::umma_commit_pair(empty_bar(s), both);      // stage (and its scales) reusable in both CTAs once these have read it
            if (last_of_set) ptx::umma_commit_pair(scales_bar(set), leader);
          }
          __syncwarp();
          if (last_of_set) {
            set ^= 1;
            if (set == 0) set_ph ^= 1u;
          }
          if (++s == F8_STAGES) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (!ok) break;
        if (issues) ptx::umma_commit_pair(tfull_bar(acc), both);
        __syncwarp();
        if (++acc == 2) {
          acc = 0;
          acc_ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else {
    // ===================== epilogue (warps 2..9 of both CTAs) =====================
    // Thread (quad, lane) owns row quad * 32 + lane; results leave through three staging blocks of 32 rows x 64 bytes (64-byte swizzle)
    // in turn, as TMA tile stores that clip at the tensor's bounds.
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const int r = quad * 32 + lane;
    const uint32_t block0 = staging + (uint32_t)(warp - 2) * (F8_EPI_BLOCKS * F8_BLOCK_BYTES);
    const uint32_t row_off = (uint32_t)lane * 64u, sw = (uint32_t)((lane >> 1) & 3);
    const uint64_t stream_out = ptx::l2_policy_evict_first();
    int block = 0;
    auto stage_begin = [&]() {            // the next block is free once all but the two newest stores have been read
      if (lane == 0) ptx::bulk_wait_read2();
      __syncwarp();
    };
    auto stage_put = [&](int q, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {      // 16-byte unit q of this row
      ptx::st_shared_v4(block0 + block * F8_BLOCK_BYTES + row_off + (((uint32_t)q ^ sw) << 4), a, b, c, d);
    };
    auto stage_send = [&](const CUtensorMap* to, int x, int y) {
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        ptx::tma_store_2d(to, block0 + block * F8_BLOCK_BYTES, x, y, stream_out);
        ptx::bulk_commit();
      }
      block = block == F8_EPI_BLOCKS - 1 ? 0 : block + 1;
    };
    const uint32_t leader_over = ptx::map_to_cta(over_bar, 0);
    const uint32_t leader_tempty[2] = {ptx::map_to_cta(tempty_bar(0), 0), ptx::map_to_cta(tempty_bar(1), 0)};
    int acc = 0, parity = 0, which, t;
    uint32_t acc_ph = 0, top_ph = 0;
    for (int nth = 0; f8_pick<MODE>(p, nth, pair_id, n_pairs, which, t) && !__any_sync(0xffffffffu, *abort_flag); ++nth) {
      const F8Product& of = p.of[which];
      const F8Tile ti = f8_tile<MODE>(of, t, rank);
      const int y0 = ti.row0 + quad * 32;
      const bool rows_here = ti.m_valid > quad * 32;       // warp-uniform
      // the residual of this thread's row and 128 columns, on its way while the tile is multiplied
      uint4 res[4][4];
      if (MODE != F8_GLU && of.residual != nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c0 = half * 128 + (half ? 3 - i : i) * 32;
          const __nv_bfloat16* at = of.residual + ((size_t)ti.row0 + r) * of.N + ti.col0 + c0;
#pragma unroll
          for (int q = 0; q < 4; ++q)
            res[i][q] = r < ti.m_valid && c0 + q * 8 < ti.n_valid ? *reinterpret_cast<const uint4*>(at + q * 8) : make_uint4(0u, 0u, 0u, 0u);
        }
      }
      if (!ptx::mbar_wait_bounded_warp(tfull_bar(acc), acc_ph, abort_flag, p.wait_limit_ns)) break;
      ptx::tc_fence_after();
      const uint32_t t_row = tmem_base + (acc ? F8_ACC1 : 0u) + ((uint32_t)(quad * 32) << 16);
      // the shared columns are the last 32 of accumulator 0 and the first 32 of accumulator 1
      const bool has_over = acc == 0 ? half == 1 : half == 0;
      auto say_over = [&]() {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster(leader_over);
      };
      if constexpr (MODE != F8_GLU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c0 = half * 128 + (half ? 3 - i : i) * 32;      // the shared columns first
          const int n_left = ti.n_valid - c0;
          const bool any = rows_here && n_left > 0;                 // warp-uniform
          float v[32];
          if (any) {
            uint32_t ra[32];
            ptx::tmem_ld32(t_row + c0, ra);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(ra[k]);
          }
          if (i == 0 && has_over) say_over();
          if (!any) continue;
          if (of.bias != nullptr) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (q * 8 < n_left) {
                Pack<__nv_bfloat16, 8> b[1];
                *reinterpret_cast<uint4*>(&b[0]) = __ldg(reinterpret_cast<const uint4*>(of.bias + ti.col0 + c0 + q * 8));
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float2 f = pair_at(b, k);
                  v[q * 8 + 2 * k] += f.x;
                  v[q * 8 + 2 * k + 1] += f.y;
                }
              }
            }
          }
          if (of.residual != nullptr) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              Pack<__nv_bfloat16, 8> b[1];
              *reinterpret_cast<uint4*>(&b[0]) = res[i][q];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 f = pair_at(b, k);
                v[q * 8 + 2 * k] += f.x;
                v[q * 8 + 2 * k + 1] += f.y;
              }
            }
          }
          if (of.out_f32) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (n_left > 16 * h) {
                stage_begin();
#pragma unroll
                for (int q = 0; q < 4; ++q)
                  stage_put(q, __float_as_uint(v[h * 16 + q * 4]), __float_as_uint(v[h * 16 + q * 4 + 1]), __float_as_uint(v[h * 16 + q * 4 + 2]),
                            __float_as_uint(v[h * 16 + q * 4 + 3]));
                stage_send(&p.maps[which].C, ti.col0 + c0 + 16 * h, ti.out_row + y0);
              }
            }
          } else {
            stage_begin();
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const Pack<__nv_bfloat16, 8> o = make_pack<__nv_bfloat16, 8>(v + q * 8);
              const uint4 w = *reinterpret_cast<const uint4*>(&o);
              stage_put(q, w.x, w.y, w.z, w.w);
            }
            stage_send(&p.maps[which].C, ti.col0 + c0, y0);
          }
        }
      } else {
        // accumulator columns 0..127 = gate, 128..255 = up; this warp: 64 of each, which with the other half's 64 share a scale
        const bool any = rows_here && ti.n_valid > 0;
        float h[64], top = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int cc = half ? 1 - i : i;                 // the shared columns first
          uint32_t rg[32], ru[32];
          if (any) {
            ptx::tmem_ld32(t_row + half * 64 + cc * 32, rg);
            ptx::tmem_ld32(t_row + 128 + half * 64 + cc * 32, ru);
            ptx::tmem_ld_wait();
          }
          if (i == 0 && has_over) say_over();
          if (any) {
            float v[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(rg[k]);
            act_values(v, p.act);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              h[i * 32 + k] = v[k] * __uint_as_float(ru[k]);
              top = larger(top, h[i * 32 + k]);
            }
          }
        }
        const bool inf = any && not_finite(top);           // rare: the maximum is taken again without
        if (inf) {
          top = 0.f;
#pragma unroll
          for (int k = 0; k < 64; ++k) top = larger_finite(top, h[k]);
        }
        s_top[parity][half][r] = top;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(top_bar(quad));
        if (!ptx::mbar_wait_bounded_warp(top_bar(quad), top_ph, abort_flag, p.wait_limit_ns)) break;
        top = fmaxf(top, s_top[parity][half ^ 1][r]);
        parity ^= 1;
        top_ph ^= 1u;
        if (any) {
          const uint32_t e = fp8_exponent(top);
          const float inv = fp8_inverse(e);
          stage_begin();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            // unit q holds columns 16q .. 16q + 15; the second half keeps its two chunks the other way round
            const int at = (q & 1) * 16, first = (q >> 1) * 32, second = 32 - first;
            float w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = half ? h[second + at + k] : h[first + at + k];
            uint32_t c[4];
            if (inf) {
#pragma unroll
              for (int k = 0; k < 4; ++k) c[k] = fp8_quad<true>(w + 4 * k, inv);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) c[k] = fp8_quad<false>(w + 4 * k, inv);
            }
            stage_put(q, c[0], c[1], c[2], c[3]);
          }
          stage_send(&p.maps[which].C, ti.col0 + half * 64, y0);
          if (half == 0 && r < ti.m_valid) p.out_scales[fp8_scale_at(ti.row0 + r, ti.col0 >> 7, fp8_atoms_across(of.N))] = (uint8_t)e;
        }
      }
      // all TMEM reads of this warp are complete (wait::ld above): hand the accumulator back
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(leader_tempty[acc]);
      if (++acc == 2) {
        acc = 0;
        acc_ph ^= 1u;
      }
    }
    if (lane == 0) ptx::bulk_wait0();   // every tile store of this warp has landed
    __syncwarp();
  }

  // ---- teardown ----
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(p.status, STATUS_TIMEOUT);
    // give copies and barrier arrivals still in flight towards either CTA's shared memory time to land
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
  }
  if (p.waits_at_end) after_previous_kernel();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync_all();      // neither CTA leaves while the other may still touch its shared memory or TMEM
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, 512);
  }
}

inline int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

template <int MODE>
cudaError_t f8_launch(const F8Params& p, cudaStream_t st) {
  static bool configured[64] = {};        // the opt-in to more than 48 KB of dynamic shared memory, once per device
  auto kern = fp8_gemm_kernel<MODE>;
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, F8_SMEM);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  const int64_t tiles = (int64_t)p.of[0].tiles + (MODE == F8_TWO ? p.of[1].tiles : 0);
  const int cap = current_sms() & ~1;
  return launch_dependent(kern, dim3((unsigned)(2 * tiles < cap ? 2 * tiles : cap)), dim3(F8_THREADS), F8_SMEM, st, p);
}

}  // namespace

bool make_fp8_maps(CUtensorMap* codes, CUtensorMap* scales, const Fp8Operand& x, int rows, int cols, uint32_t box_rows) {
  const uint64_t atoms = (uint64_t)cdiv(rows, 128) * fp8_atoms_across(cols);
  return make_tile_map(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, x.codes, rows, cols, fp8_pitch(cols), 128, box_rows, CU_TENSOR_MAP_SWIZZLE_128B) &&
         make_tile_map(scales, CU_TENSOR_MAP_DATA_TYPE_INT32, 4, x.scales, atoms, 128, 128, 128, 1, CU_TENSOR_MAP_SWIZZLE_NONE);
}

namespace {

bool f8_linear(const Fp8Gemm& g, F8Maps* m, F8Product* of) {
  *of = {};
  of->M = g.M; of->N = g.N; of->K = g.K;
  of->tiles_m = cdiv(g.M, F8_PM);
  of->tiles_n = cdiv(g.N, F8_BN);
  of->across = (int)fp8_atoms_across(g.K);
  of->pieces = 1;
  of->piece_steps = cdiv(g.K, F8_BK);
  of->bias = static_cast<const __nv_bfloat16*>(g.bias);
  of->residual = static_cast<const __nv_bfloat16*>(g.residual);
  of->out_f32 = g.out_f32;
  if (g.pieces > 1) {
    of->pieces = g.pieces;
    of->piece_steps = g.piece_steps;
    of->piece_rows = fp8_piece_rows(g.M);
  }
  of->tiles = of->tiles_m * of->tiles_n * of->pieces;
  return make_fp8_maps(&m->A, &m->SA, g.A, g.M, g.K, F8_BM) && make_fp8_maps(&m->B, &m->SB, g.B, g.N, g.K, F8_BNH) &&
         (g.out_f32 ? make_tile_map(&m->C, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, g.C, of->pieces > 1 ? (uint64_t)of->pieces * of->piece_rows : g.M, g.N, g.N,
                                    16, 32, CU_TENSOR_MAP_SWIZZLE_64B)
                    : make_tile_map(&m->C, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, g.C, g.M, g.N, g.N, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B));
}
F8Params f8_params(const Fp8Gemm& g) {
  F8Params p;
  p.of[1] = {};
  p.ahead = 0;
  p.act = g.act;
  p.out_scales = static_cast<uint8_t*>(g.out_scales);
  p.status = g.status;
  p.wait_limit_ns = DEFAULT_WAIT_LIMIT_NS;
  p.waits_at_end = g.waits_at_end;
  return p;
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8Gemm& g, cudaStream_t st) {
  F8Params p = f8_params(g);
  if (!g.B1.codes) return f8_linear(g, &p.maps[0], &p.of[0]) ? f8_launch<F8_LINEAR>(p, st) : cudaErrorInvalidValue;
  F8Product& of = p.of[0];
  of = {};
  of.M = g.M; of.N = g.N; of.K = g.K;
  of.tiles_m = cdiv(g.M, F8_PM);
  of.tiles_n = cdiv(g.N, F8_BNH);
  of.across = (int)fp8_atoms_across(g.K);
  of.pieces = 1;
  of.piece_steps = cdiv(g.K, F8_BK);
  of.tiles = of.tiles_m * of.tiles_n;
  F8Maps& m = p.maps[0];
  // the columns up to the pitch are written too
  const bool ok = make_fp8_maps(&m.A, &m.SA, g.A, g.M, g.K, F8_BM) && make_fp8_maps(&m.B, &m.SB, g.B, g.N, g.K, F8_BNH) &&
                  make_fp8_maps(&p.maps[1].B, &p.maps[1].SB, g.B1, g.N, g.K, F8_BNH) &&
                  make_tile_map(&m.C, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, g.C, g.M, fp8_pitch(g.N), fp8_pitch(g.N), 64, 32, CU_TENSOR_MAP_SWIZZLE_64B);
  return ok ? f8_launch<F8_GLU>(p, st) : cudaErrorInvalidValue;
}

cudaError_t launch_fp8_gemms(const Fp8Gemm& a, const Fp8Gemm& b, cudaStream_t st) {
  F8Params p = f8_params(a);
  if (!f8_linear(a, &p.maps[0], &p.of[0]) || !f8_linear(b, &p.maps[1], &p.of[1])) return cudaErrorInvalidValue;
  p.ahead = fp8_tile_cost(p.of[0].piece_steps) / fp8_tile_cost(p.of[1].piece_steps);
  return f8_launch<F8_TWO>(p, st);
}

}  // namespace grouter
