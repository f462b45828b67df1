// Per-expert counts, the router's balance and z losses, and the gradient of its scores.
//
//   c_e  = #{(t, j): idx[t,j] = e, token t counts}         f_e = E c_e / sum_e' c_e'         n = tokens that count
//   p_te = softmax of row t of the scores                   lse_t = log sum_e exp s_te
//   balance = sum_e f_e (1/n) sum_t p_te = (1/n) sum_t a_t      with a_t = sum_e f_e p_te
//   z       = (1/n) sum_t lse_t^2                               loss = ca balance + cz z
//   d loss / d s_te = (ca/n) p_te (f_e - a_t) + (2 cz/n) lse_t p_te              (the counts do not depend on the scores)
// and, joined in the same pass, what comes back through the gates r(x) = g(kept scores):
//   softmax over the kept k: q_j (dg_j - sum_i q_i dg_i)        sigmoid of each: q_j (1 - q_j) dg_j
//
// The counts are known before the scores are read, so the loss needs no column sums of p: one number a token (a_t) carries
// it, and one pass over the scores gives the loss and its gradient.  Bound by HBM: scores read once, gradient written once.
// Neighbouring lanes hold a token's row in registers, 16 bytes at a time; a block's token sums are added in a fixed
// order, and the last step (one block) adds the blocks' sums in double precision.
//
// Measured: 1048575 tokens x 256 bf16 with a mask 190 us for losses and gradient (5.65 TB/s of 6.46), the counts 17 us before
// them; 32768 x 128 f32 with the gates' gradient 21-22 us in all; 511 tokens 8.8 us (two launches).
// With the gates' gradient wide routers are bound by registers and shared memory, not by HBM: 524288 x 160 bf16 194 us with the counts
// (99 without gates), 1048575 x 60 148 us, 200000 x 333 154 us, each 3.4 to 3.6 times their bytes at a plain copy's pace.
//
// A score of -inf takes its expert out (p = 0, no gradient).  A row of nothing but -inf has p = 0 throughout and no
// z-loss term.  A token whose mask byte is zero contributes nothing and gets a zero gradient row, whatever its scores are.
#include <cooperative_groups.h>
#include <math.h>

#include "vec.cuh"

namespace grouter {

constexpr int BAL_THREADS = 256;
constexpr int BAL_WARPS = BAL_THREADS / 32;
constexpr int BAL_MAX_E = 1024;
constexpr int COUNT_THREADS = 1024;
constexpr int COUNT_CLUSTER = 8;
// Up to this many ids one cluster counts them all and writes the sums itself: one launch instead of two zeroings and a kernel.
constexpr uint32_t COUNT_CLUSTER_SLOTS = 1 << 19;
constexpr int COUNT_SLOTS = 4224;       // counters a block of the histogram keeps: 32 copies of 128 experts and of two more

// Histogram of the ids.  A thread takes 16 bytes of ids at a time (IPT of them).  Lanes spread over `copies` (a power of two up to
// 32) copies of the counters, the copies of one expert side by side: with 32 of them every lane has a bank of its own, whatever
// the ids are.  Two counters more, E and E + 1, take the ids that are out of range and those of masked tokens: no id is a branch.
// CLUSTER: the grid is one cluster of COUNT_CLUSTER blocks, which add up their counters through each other's shared memory and
// store the sums; otherwise any number of blocks adds to outputs that were zeroed before.
template <typename Id, bool CLUSTER>
__global__ void __launch_bounds__(COUNT_THREADS) expert_counts_kernel(const Id* __restrict__ idx, uint32_t slots, uint32_t k, int E,
                                                                      int copies, const uint8_t* __restrict__ mask,
                                                                      int32_t* __restrict__ counts, int32_t* __restrict__ n_tokens,
                                                                      int32_t* __restrict__ status) {
  constexpr int IPT = 16 / (int)sizeof(Id);
  __shared__ int32_t s_cnt[COUNT_SLOTS];
  __shared__ int32_t s_sum[BAL_MAX_E + 2];        // this block's counts
  __shared__ int32_t s_tokens;
  const int rows = E + 2;
  for (int i = threadIdx.x; i < rows * copies; i += COUNT_THREADS) s_cnt[i] = 0;
  if (threadIdx.x == 0) s_tokens = mask == nullptr && blockIdx.x == 0 ? (int32_t)(slots / k) : 0;      // without a mask: all tokens
  __syncthreads();
  int32_t* mine = s_cnt + (threadIdx.x & (copies - 1));
  int tokens = 0;
  const uint32_t stride = gridDim.x * COUNT_THREADS * IPT;      // slots + stride < 2^32: slots < 2^31, stride < 2^24
  struct Piece {
    alignas(16) Id ids[IPT];
  };
  auto load = [&](uint32_t s0) {
    Piece r;
    if (s0 + IPT <= slots) {
      *reinterpret_cast<uint4*>(r.ids) = ld_stream16(idx + s0);
    } else {
#pragma unroll
      for (int i = 0; i < IPT; ++i) r.ids[i] = s0 + i < slots ? idx[s0 + i] : Id(0);
    }
    return r;
  };
  uint32_t s0 = (blockIdx.x * COUNT_THREADS + threadIdx.x) * IPT;
  Piece next = load(s0);
  for (; s0 < slots; s0 += stride) {
    const Piece cur = next;
    next = load(s0 + stride);                                   // on its way while these are counted
    if (mask == nullptr && s0 + IPT <= slots) {                 // every id counts: no need to know whose it is
#pragma unroll
      for (int i = 0; i < IPT; ++i) atomicAdd(mine + min((uint32_t)cur.ids[i], (uint32_t)E) * copies, 1);
      continue;
    }
    uint32_t t = s0 / k, j = s0 - t * k;
    bool live = mask == nullptr || mask[t] != 0;
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
      if (s0 + i < slots) {
        tokens += live && j == 0 && mask != nullptr;
        atomicAdd(mine + (live ? min((uint32_t)cur.ids[i], (uint32_t)E) : (uint32_t)E + 1) * copies, 1);
        if (++j == k) {
          j = 0;
          ++t;
          if (mask != nullptr && s0 + i + 1 < slots) live = mask[t] != 0;
        }
      }
    }
  }
  if (tokens) atomicAdd(&s_tokens, tokens);
  __syncthreads();
  // `copies` neighbouring lanes add up an expert
  for (int i0 = 0; i0 < rows * copies; i0 += COUNT_THREADS) {
    const int i = i0 + threadIdx.x;
    int32_t c = i < rows * copies ? s_cnt[i] : 0;
    for (int o = copies / 2; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    if (i < rows * copies && (i & (copies - 1)) == 0) s_sum[i / copies] = c;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    if (s_sum[E] != 0 && status) atomicOr(status, STATUS_BAD_INDEX);
    s_sum[E] = s_tokens;
  }
  if constexpr (CLUSTER) {
    cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
    cl.sync();
    for (int e = cl.block_rank() * COUNT_THREADS + threadIdx.x; e <= E; e += COUNT_CLUSTER * COUNT_THREADS) {
      int32_t c = 0;
#pragma unroll
      for (int r = 0; r < COUNT_CLUSTER; ++r) c += cl.map_shared_rank(s_sum, r)[e];
      if (e < E) counts[e] = c;
      else *n_tokens = c;
    }
    cl.sync();                                    // nobody leaves while its counters are read
  } else {
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += COUNT_THREADS) {
      const int32_t c = s_sum[e];
      if (c) atomicAdd(e < E ? counts + e : n_tokens, c);
    }
  }
}

struct BalanceParams {
  const void* logits;
  int64_t ld;
  const void* idx;
  int idx_i32;
  const uint8_t* mask;
  const int32_t *counts, *n_tokens;
  const float* dgates;
  int sigmoid;
  int T, E, k;
  float ca, cz;
  const float* dloss;
  float* loss;
  void* dlogits;
  double2* partial;     // [blocks] sums of a_t and lse_t^2 (loss wanted)
  int32_t* status;
};

__device__ __forceinline__ void write_loss(const BalanceParams& p, double a, double z, int n) {
  const double per = n > 0 ? 1.0 / (double)n : 0.0;
  const float balance = (float)(a * per), zl = (float)(z * per);
  // a loss that does not count (coefficient zero) does not spoil the sum either when it is not finite
  p.loss[0] = (p.ca != 0.f ? p.ca * balance : 0.f) + (p.cz != 0.f ? p.cz * zl : 0.f);
  p.loss[1] = balance;
  p.loss[2] = zl;
}

// 2^d by the hardware's exponential (within 2 ulp of f32: the gradient of f32 scores is as close to the 64-bit definition as plain f32
// operations come, 8e-8 of it); results below the normal range of f32 are zero
__device__ __forceinline__ float exp2_of(float d) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  return r;
}
__device__ __forceinline__ float exp_of(float d) { return exp2_of(d * 1.4426950408889634f); }
// the largest of three (a NaN only if all are)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Rounds whose scores a thread has on their way or in use: 96 to 256 bytes of them.
__host__ __device__ constexpr int balance_ring(int bytes, int epl) { return bytes * epl >= 64 ? (bytes * epl >= 128 ? 2 : 3) : bytes * epl >= 32 ? 4 : 6; }

// LPT neighbouring lanes hold a token's row, EPL elements each, VE to an access.  Few lanes and many elements: the three
// reductions over a row cost log2(LPT) shuffles each for a whole warp's 32 / LPT tokens, which is what bounded one warp a token
// (326 instructions a token of 256 scores).  The arithmetic is done two elements to an instruction where there is one for it.
// Blocks are resident and walk over the tokens; the scores of the next rounds are on their way into shared memory (one round ahead
// in registers was 24 KB an SM and 3.8 TB/s), every thread copying and reading back its own, so that no barrier is needed.
// Dynamic shared memory: that ring, f [E], then (with dgates) one row of E sums for every lane group, zero between tokens.
template <typename T, int VE, int LPT, int EPL, bool GATES>
__global__ void __launch_bounds__(BAL_THREADS) balance_kernel(const BalanceParams p) {
  constexpr bool RING = VE > 1;                       // rows that are not 16-byte aligned: plain loads, one round ahead
  constexpr int S = balance_ring(sizeof(T), EPL);
  extern __shared__ uint4 s_dyn[];
  Pack<T, VE>* s_ring = reinterpret_cast<Pack<T, VE>*>(s_dyn);      // RING: [S][NV][BAL_THREADS]
  float* s_f = reinterpret_cast<float*>(s_ring + (RING ? S * (EPL / VE) * BAL_THREADS : 0));
  __shared__ double s_part[2][BAL_WARPS];
  __shared__ unsigned long long s_count[BAL_WARPS];
  constexpr int NV = EPL / VE, PAIRS = EPL / 2;
  constexpr int TPW = 32 / LPT;                       // tokens a warp works on at a time
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sl = lane & (LPT - 1), grp = lane / LPT;
  const int E = p.E, epad = (E + 3) & ~3;

  // Columns beyond E are never loaded and stay -inf: p = 0.  What a masked token's row holds is computed along and dropped.
  Pack<T, VE> q[NV];
#pragma unroll
  for (int n = 0; n < NV; ++n)
#pragma unroll
    for (int i = 0; i < VE; ++i) q[n].v[i] = from_f32<T>(-INFINITY);
  auto slot = [&](int s, int n) { return s_ring + (s * NV + n) * BAL_THREADS + threadIdx.x; };
  auto fetch = [&](int64_t t, int s) {
    if (t < p.T) {
      const T* row = reinterpret_cast<const T*>(p.logits) + t * p.ld;
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const int c = (n * LPT + sl) * VE;
        if (c < E) {
          if constexpr (RING && VE * sizeof(T) == 16) copy16_async(slot(s, n), row + c);
          else if constexpr (RING) copy8_async(slot(s, n), row + c);
          else q[n] = ld_pack<T, VE>(row + c);
        }
      }
    }
    if constexpr (RING) copies_commit();
  };
  // What else a lane needs of its token: whether it counts, and (GATES, lane j < k of the group: LPT >= k) its j-th kept expert with
  // the gradient of its gate, two rounds ahead, and that expert's score one round ahead.
  // All of it as loaded: whatever is computed from it here would wait for it here.
  struct Side {
    int e, mask;
    float dg;
  };
  auto side = [&](int64_t t) {
    Side r{-1, 0, 0.f};
    if (t < p.T) {
      r.mask = 1;
      if (p.mask != nullptr) r.mask = __ldg(p.mask + t);
      if (GATES && sl < p.k) {
        const int64_t at = t * p.k + sl;
        r.e = p.idx_i32 ? __ldg(reinterpret_cast<const int32_t*>(p.idx) + at) : (int)__ldg(reinterpret_cast<const uint8_t*>(p.idx) + at);
        r.dg = __ldg(p.dgates + at);
      }
    }
    return r;
  };
  auto score = [&](int64_t t, const Side& r) {
    T s = from_f32<T>(-INFINITY);
    if (GATES && r.mask != 0 && sl < p.k && (unsigned)r.e < (unsigned)E) s = reinterpret_cast<const T*>(p.logits)[t * p.ld + r.e];
    return s;
  };

  const int64_t step = (int64_t)gridDim.x * BAL_WARPS * TPW;
  int64_t t = ((int64_t)blockIdx.x * BAL_WARPS + warp) * TPW + grp;
  if constexpr (RING) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
        if ((n * LPT + sl) * VE >= E) *slot(s, n) = q[n];
      fetch(t + s * step, s);
    }
  } else {
    fetch(t, 0);
  }
  Side next = side(t), after = side(t + step);
  T next_s = score(t, next);

  // f_e = E c_e / sum c, and a row of zeros for every lane group
  {
    unsigned long long sum = 0;                       // counts may come summed over many ranks
    for (int e = threadIdx.x; e < E; e += BAL_THREADS) {
      const unsigned c = (unsigned)__ldg(p.counts + e);
      s_f[e] = (float)c;
      sum += c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_count[warp] = sum;
  }
  float* s_gate = s_f + epad + (size_t)(warp * TPW + grp) * epad;
  if (GATES)
    for (int e = sl; e < E; e += LPT) s_gate[e] = 0.f;
  __syncthreads();
  unsigned long long total = 0;
#pragma unroll
  for (int w = 0; w < BAL_WARPS; ++w) total += s_count[w];
  const float per_count = total > 0 ? (float)E / (float)total : 0.f;
  // a lane's elements in pairs: pair j holds elements 2j and 2j + 1 of its [NV][VE]
  auto col = [&](int k) { return ((k / VE) * LPT + sl) * VE + k % VE; };
  float2 f[PAIRS];
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) {
    f[j].x = col(2 * j) < E ? s_f[col(2 * j)] * per_count : 0.f;
    f[j].y = col(2 * j + 1) < E ? s_f[col(2 * j + 1)] * per_count : 0.f;
  }
  const int n_tok = __ldg(p.n_tokens);
  const float per = n_tok > 0 ? 1.f / (float)n_tok : 0.f;
  const float up = p.dloss ? __ldg(p.dloss) : 1.f;
  const float ka = p.ca * per * up, kz = 2.f * p.cz * per * up;
  float sum_a = 0.f, sum_z = 0.f;

  int s_at = 0;
  for (; t - grp < p.T; t += step) {                  // the warp's tokens start at t - grp: the same trips for all its lanes
    const bool here = t < p.T, live = next.mask != 0;
    const int e = next.e;
    const float dg = next.dg, s = to_f32(next_s);     // GATES: of this lane's slot
    next = after;
    next_s = score(t + step, next);
    after = side(t + 2 * step);
    if constexpr (RING) {
      copies_wait<S - 1>();
#pragma unroll
      for (int n = 0; n < NV; ++n) q[n] = *slot(s_at, n);
    }
    float2 v[PAIRS];
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) v[j] = pair_at(q, j);
    if constexpr (!RING) fetch(t + step, 0);
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) top = max3(top, v[j].x, v[j].y);
    const bool kept = GATES && live && sl < p.k;
    const bool ok = kept && (unsigned)e < (unsigned)E;
    if (GATES && kept && !ok && p.status) atomicOr(p.status, STATUS_BAD_INDEX);
    top = lanes_max<LPT>(top);
    const bool some = top != -INFINITY;
    const float base = some ? top : 0.f;              // a row without a score: every exp below is 0
    float2 z2 = both(0.f), a2 = both(0.f);
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      // the difference first: its rounding is relative to it, and scores of any size stay in range
      const float2 d = mul2(add2(v[j], both(-base)), both(1.4426950408889634f));
      v[j] = make_float2(exp2_of(d.x), exp2_of(d.y));
      z2 = add2(z2, v[j]);
      a2 = fma2(v[j], f[j], a2);
    }
    float z = z2.x + z2.y, a = a2.x + a2.y;
    if constexpr (RING) {                             // the slot has been read: v comes from it
      fetch(t + S * step, s_at);
      s_at = s_at + 1 == S ? 0 : s_at + 1;
    }
    z = lanes_sum<LPT>(z);
    a = lanes_sum<LPT>(a);
    const float inv_z = some ? 1.f / z : 0.f;
    const float lse = some ? base + __logf(z) : z;            // z >= 1: within 2^-21.  No score: z = 0, or NaN if there was one
    a *= inv_z;
    if (sl == 0 && live) {
      sum_a += a;
      sum_z += lse * lse;
    }
    if (p.dlogits == nullptr) continue;
    if (GATES) {
      float back;
      if (p.sigmoid) {
        // q (1 - q) with 1 - q = 1 / (1 + exp(s)), not by subtraction
        const float x = exp_of(-fabsf(s));
        back = x / ((1.f + x) * (1.f + x)) * dg;
      } else {
        const float m = lanes_max<LPT>(s);
        const float q = s == -INFINITY ? 0.f : exp_of(s - m);
        const float qs = lanes_sum<LPT>(q), qd = lanes_sum<LPT>(ok ? q * dg : 0.f);
        const float inv = qs > 0.f || qs != qs ? 1.f / qs : 0.f;
        back = q * inv * (dg - qd * inv);
      }
      // The slots' terms meet the row's elements in shared memory.  Where a token names an expert twice (ids folded after the
      // choice), the first of its slots brings the sum, added up in slot order.
      const unsigned same = __match_any_sync(0xffffffffu, ok ? (grp << 16) + e : (1 << 30) + lane);
      if (__any_sync(0xffffffffu, (same & (same - 1)) != 0)) {
        const float mine = back;
        back = 0.f;
        for (int j = 0; j < 32; ++j) {
          const float other = __shfl_sync(0xffffffffu, mine, j);
          if (same >> j & 1) back += other;
        }
      }
      if (ok && lane == __ffs(same) - 1) s_gate[e] = back;
      __syncwarp();
    }
    T* out = reinterpret_cast<T*>(p.dlogits) + t * E;
    // p (ka (f - a) + kz lse) = v (k1 f + k0)
    const float2 k1 = both(inv_z * ka), k0 = both(inv_z * (kz * lse - ka * a));
    float o[EPL];
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      const float2 d = mul2(v[j], fma2(k1, f[j], k0));
      o[2 * j] = d.x;
      o[2 * j + 1] = d.y;
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * LPT + sl) * VE;
      if (here && c < E) {
        float w[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) w[i] = o[n * VE + i];
        if (GATES) {
          if constexpr (VE == 1) {
            w[0] += s_gate[c];
          } else {
#pragma unroll
            for (int i = 0; i < VE; i += 4) {
              const float4 g = *reinterpret_cast<const float4*>(s_gate + c + i);
              w[i] += g.x;
              w[i + 1] += g.y;
              w[i + 2] += g.z;
              w[i + 3] += g.w;
            }
          }
        }
        Pack<T, VE> r = make_pack<T, VE>(w);
        if (!live) r = Pack<T, VE>{};                 // zeros
        *reinterpret_cast<Pack<T, VE>*>(out + c) = r;
      }
    }
    if (GATES) {
      __syncwarp();
      if (ok) s_gate[e] = 0.f;
      __syncwarp();
    }
  }
  if (p.loss == nullptr) return;
  let_next_kernel_start();
  sum_a = lanes_sum<32>(sum_a);
  sum_z = lanes_sum<32>(sum_z);
  if (lane == 0) {
    s_part[0][warp] = sum_a;
    s_part[1][warp] = sum_z;
  }
  __syncthreads();
  __shared__ double2 s_sum;
  if (threadIdx.x == 0) {
    double a = 0, z = 0;
    for (int w = 0; w < BAL_WARPS; ++w) {
      a += s_part[0][w];
      z += s_part[1][w];
    }
    s_sum = make_double2(a, z);
  }
  cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
  if (cl.num_blocks() == gridDim.x) {                 // the whole grid is one cluster: its blocks add up among themselves
    cl.sync();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      double a = 0, z = 0;
      for (unsigned r = 0; r < gridDim.x; ++r) {
        const double2 v = *cl.map_shared_rank(&s_sum, r);
        a += v.x;
        z += v.y;
      }
      write_loss(p, a, z, n_tok);
    }
    cl.sync();                                        // nobody leaves while its sums are read
  } else if (threadIdx.x == 0) {
    p.partial[blockIdx.x] = s_sum;
  }
}

__global__ void __launch_bounds__(256) balance_finish_kernel(const BalanceParams p, int n_part) {
  __shared__ double s[2][256];
  double a = 0, z = 0;
  after_previous_kernel();
  for (int i = threadIdx.x; i < n_part; i += 256) {
    const double2 v = p.partial[i];
    a += v.x;
    z += v.y;
  }
  s[0][threadIdx.x] = a;
  s[1][threadIdx.x] = z;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) {
      s[0][threadIdx.x] += s[0][threadIdx.x + o];
      s[1][threadIdx.x] += s[1][threadIdx.x + o];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) write_loss(p, s[0][0], s[1][0], __ldg(p.n_tokens));
}

namespace {

constexpr int BAL_MAX_BLOCKS = 1184;   // 148 SMs x 8 blocks
constexpr int BAL_CLUSTER = 8;         // a grid of up to so many blocks is one cluster, and needs neither workspace nor second kernel

// Lanes a token: enough for 16 elements each and for one of the kept experts each.  (With or without gates: the sums of a row then
// run in the same order, and while one round of blocks holds all tokens the losses are the same bits.)
int balance_lanes(int E, int k) {
  int lpt = 1;
  while (lpt < 32 && (lpt * 16 < E || lpt < k)) lpt *= 2;
  return lpt;
}
int64_t balance_blocks(int T, int E, int k) {
  const int per_block = BAL_WARPS * (32 / balance_lanes(E, k));
  return ((int64_t)T + per_block - 1) / per_block;
}

template <typename Id>
cudaError_t count_in_cluster(const Id* idx, uint32_t slots, uint32_t k, int E, int copies, const uint8_t* mask, int32_t* counts, int32_t* n_tokens,
                             int32_t* status, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(COUNT_CLUSTER);
  cfg.blockDim = dim3(COUNT_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = COUNT_CLUSTER;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, expert_counts_kernel<Id, true>, idx, slots, k, E, copies, mask, counts, n_tokens, status);
}

template <typename T, int VE, int LPT, int EPL, bool GATES>
cudaError_t balance_launch_g(const BalanceParams& p, cudaStream_t st) {
  constexpr int TPB = BAL_WARPS * (32 / LPT);
  const int epad = (p.E + 3) & ~3;
  constexpr int RING = VE > 1 ? balance_ring(sizeof(T), EPL) * EPL * (int)sizeof(T) * BAL_THREADS : 0;      // at most 64 KB
  constexpr int MAX_SMEM = RING + (int)sizeof(float) * LPT * EPL * (1 + (GATES ? TPB : 0));                // E <= LPT * EPL: 37 KB more
  const size_t smem = RING + sizeof(float) * epad * (1 + (GATES ? TPB : 0));
  auto kern = balance_kernel<T, VE, LPT, EPL, GATES>;
  const int64_t want = balance_blocks(p.T, p.E, p.k);
  static int resident[64] = {};       // blocks an SM holds, which is what walks over the tokens; asked once per device
  int dev = 0, per_sm = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64) per_sm = resident[dev];
  if (per_sm == 0) {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, BAL_THREADS, MAX_SMEM);
    if (e != cudaSuccess) return e;
    if (per_sm < 1) per_sm = 1;
    if (dev >= 0 && dev < 64) resident[dev] = per_sm;
  }
  int cap = current_sms() * per_sm;
  if (cap > BAL_MAX_BLOCKS) cap = BAL_MAX_BLOCKS;
  const int grid = (int)(want < cap ? want : cap);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(BAL_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = grid;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = p.loss && grid <= BAL_CLUSTER ? 1 : 0;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
  if (e == cudaSuccess && p.loss && grid > BAL_CLUSTER) e = launch_dependent(balance_finish_kernel, dim3(1), dim3(256), 0, st, p, grid);
  return e;
}

template <typename T, int VE, int LPT, int EPL>
cudaError_t balance_launch(const BalanceParams& p, cudaStream_t st) {
  return p.dgates ? balance_launch_g<T, VE, LPT, EPL, true>(p, st) : balance_launch_g<T, VE, LPT, EPL, false>(p, st);
}

template <typename T, int VE, int EPL>
cudaError_t balance_by_lanes(const BalanceParams& p, int lpt, cudaStream_t st) {
  switch (lpt) {
    case 1: return balance_launch<T, VE, 1, EPL>(p, st);
    case 2: return balance_launch<T, VE, 2, EPL>(p, st);
    case 4: return balance_launch<T, VE, 4, EPL>(p, st);
    case 8: return balance_launch<T, VE, 8, EPL>(p, st);
    case 16: return balance_launch<T, VE, 16, EPL>(p, st);
    default: return balance_launch<T, VE, 32, EPL>(p, st);
  }
}

template <typename T, int VE>
cudaError_t balance_by_width(const BalanceParams& p, cudaStream_t st) {
  const int lpt = balance_lanes(p.E, p.k);
  if (lpt * 16 < p.E) return balance_launch<T, VE, 32, 32>(p, st);
  if constexpr (VE > 1) {
    if (lpt * 8 >= p.E) return balance_by_lanes<T, VE, 8>(p, lpt, st);
  }
  return balance_by_lanes<T, VE, 16>(p, lpt, st);
}

}  // namespace
}  // namespace grouter

using namespace grouter;

extern "C" {

int grouter_expert_counts(const void* idx, int32_t idx_dtype, const uint8_t* mask, int32_t T, int32_t k, int32_t E, int32_t* counts,
                          int32_t* n_tokens, int32_t* status, void* stream) {
  if (!counts || !n_tokens || T < 0 || k < 1 || E < 1 || (T > 0 && !idx)) return GROUTER_ERR_INVALID_ARG;
  if (idx_dtype != GROUTER_IDX_U8 && idx_dtype != GROUTER_IDX_I32) return GROUTER_ERR_INVALID_ARG;
  if (E > BAL_MAX_E || k > 32 || (int64_t)T * k > INT32_MAX || (idx_dtype == GROUTER_IDX_U8 && E > 256)) return GROUTER_ERR_UNSUPPORTED;
  if (!aligned_to(idx, 16) || !aligned_to(counts, 4) || !aligned_to(n_tokens, 4) || !aligned_to(status, 4)) return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint32_t slots = (uint32_t)T * (uint32_t)k;
  const bool u8 = idx_dtype == GROUTER_IDX_U8;
  int copies = 32;
  while (copies * (E + 2) > COUNT_SLOTS) copies /= 2;
  cudaError_t e;
  if (slots <= COUNT_CLUSTER_SLOTS) {
    e = u8 ? count_in_cluster(static_cast<const uint8_t*>(idx), slots, k, E, copies, mask, counts, n_tokens, status, st)
           : count_in_cluster(static_cast<const int32_t*>(idx), slots, k, E, copies, mask, counts, n_tokens, status, st);
  } else {
    if (cudaMemsetAsync(counts, 0, sizeof(int32_t) * E, st) != cudaSuccess || cudaMemsetAsync(n_tokens, 0, sizeof(int32_t), st) != cudaSuccess)
      return GROUTER_ERR_CUDA;
    const int64_t per_block = (int64_t)COUNT_THREADS * (u8 ? 16 : 4), want = ((int64_t)slots + per_block - 1) / per_block;
    const int cap = current_sms() * 2, grid = (int)(want < cap ? want : cap);
    if (u8)
      expert_counts_kernel<uint8_t, false><<<grid, COUNT_THREADS, 0, st>>>(static_cast<const uint8_t*>(idx), slots, k, E, copies, mask, counts,
                                                                          n_tokens, status);
    else
      expert_counts_kernel<int32_t, false><<<grid, COUNT_THREADS, 0, st>>>(static_cast<const int32_t*>(idx), slots, k, E, copies, mask, counts,
                                                                          n_tokens, status);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

size_t grouter_balance_loss_workspace_bytes(int32_t T, int32_t E, int32_t k) {
  if (T < 1 || E < 1 || k < 1 || balance_blocks(T, E, k) <= BAL_CLUSTER) return 0;
  return sizeof(double2) * BAL_MAX_BLOCKS;
}

int grouter_balance_loss(const void* logits, int64_t ld, int32_t dtype, const void* idx, int32_t idx_dtype, const uint8_t* mask,
                         const int32_t* counts, const int32_t* n_tokens, const float* dgates, int32_t norm, int32_t T, int32_t E, int32_t k,
                         float balance_coef, float z_coef, const float* dloss, float* loss, void* dlogits, void* workspace, int32_t* status,
                         void* stream) {
  if (!counts || !n_tokens || T < 0 || E < 1 || k < 1 || ld < E || (!loss && !dlogits)) return GROUTER_ERR_INVALID_ARG;
  if (T > 0 && (!logits || (dgates && (!idx || !dlogits)))) return GROUTER_ERR_INVALID_ARG;
  if ((dtype != GROUTER_BF16 && dtype != GROUTER_F32) || (idx_dtype != GROUTER_IDX_U8 && idx_dtype != GROUTER_IDX_I32) ||
      (norm != GROUTER_NORM_SOFTMAX && norm != GROUTER_NORM_SIGMOID))
    return GROUTER_ERR_INVALID_ARG;
  if (E > BAL_MAX_E || k > 32 || (int64_t)T * k > INT32_MAX || T > INT32_MAX - (1 << 20) || (idx && idx_dtype == GROUTER_IDX_U8 && E > 256))
    return GROUTER_ERR_UNSUPPORTED;
  if (loss && !workspace && grouter_balance_loss_workspace_bytes(T, E, k) > 0) return GROUTER_ERR_INVALID_ARG;
  const size_t el = dtype == GROUTER_F32 ? 4 : 2;
  if (!aligned_to(logits, el) || !aligned_to(dlogits, el) || !aligned_to(dgates, 4) || !aligned_to(counts, 4) || !aligned_to(n_tokens, 4) ||
      !aligned_to(dloss, 4) || !aligned_to(loss, 4) || !aligned_to(status, 4) || !aligned_to(workspace, 16) ||
      (idx_dtype == GROUTER_IDX_I32 && !aligned_to(idx, 4)))
    return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    if (loss && cudaMemsetAsync(loss, 0, 3 * sizeof(float), st) != cudaSuccess) return GROUTER_ERR_CUDA;
    return GROUTER_OK;
  }
  BalanceParams p{};
  p.logits = logits; p.ld = ld; p.idx = idx; p.idx_i32 = idx_dtype == GROUTER_IDX_I32; p.mask = mask; p.counts = counts; p.n_tokens = n_tokens;
  p.dgates = dgates; p.sigmoid = norm == GROUTER_NORM_SIGMOID; p.T = T; p.E = E; p.k = k; p.ca = balance_coef; p.cz = z_coef; p.dloss = dloss;
  p.loss = loss; p.dlogits = dlogits; p.partial = static_cast<double2*>(workspace); p.status = status;
  // 16-byte accesses where every row starts on a 16-byte boundary (8-byte ones for bf16 on such a boundary: 60 experts), single
  // elements otherwise
  const int ve = dtype == GROUTER_F32 ? vec16<float>() : vec16<__nv_bfloat16>();
  const bool vec = E % ve == 0 && ld % ve == 0 && aligned_to(logits, 16) && aligned_to(dlogits, 16);
  cudaError_t e;
  if (dtype == GROUTER_F32) e = vec ? balance_by_width<float, vec16<float>()>(p, st) : balance_by_width<float, 1>(p, st);
  else if (vec) e = balance_by_width<__nv_bfloat16, vec16<__nv_bfloat16>()>(p, st);
  else if (E % 4 == 0 && ld % 4 == 0 && aligned_to(logits, 8) && aligned_to(dlogits, 8)) e = balance_by_width<__nv_bfloat16, 4>(p, st);
  else e = balance_by_width<__nv_bfloat16, 1>(p, st);
  return e == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
