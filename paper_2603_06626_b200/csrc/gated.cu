// Gated feed-forward block, and the linear layer in 8 bits: the calls around their products.
//
//   forward    p = x W_gu^T = [g | u]     h = act(g) u     y = h W_d^T + r          x [T,d], W_gu [2H,d], W_d [d,H]
//   backward   dh = dy W_d     du = dh act(g)     dg = dh u act'(g)     dp = [dg | du]
//              dx = dp W_gu     dW_gu = dp^T x     dW_d = dy^T h
//   8 bits     the same forward pass on codes and scales (fp8.cuh), h leaving as codes: y = q(act(q(x) Wg^T) (q(x) Wu^T)) Wd^T + r
//   linear     y = q(x) q(W)^T + b + r     dx = q(dy) q(W)     dW = q(dy^T) q(x^T)^T     db = sum_t dy_t
//
// Both projections, the activation and the product are one kernel (gemm.cu, MODE_GLU; fp8_gemm.cu, F8_GLU): a tile holds 128 gate and the
// 128 up columns that belong to them, so h is formed on the accumulators.  dh never leaves the chip either: its product's epilogue
// (MODE_GLU_BACK) writes dp and h, which is cheaper to form again from p than to keep.
#include "fp8.cuh"
#include "fp8_gemm.cuh"

namespace grouter {
namespace {

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline bool fits_int(int64_t v) { return v <= INT32_MAX - 256; }

struct GatedWorkspace {
  size_t dp, h, pieces_gu, pieces_d, bytes;
};
GatedWorkspace gated_workspace(int T, int d, int H) {
  GatedWorkspace w{};
  w.h = up256((size_t)T * 2 * H * 2);
  w.pieces_gu = w.h + up256((size_t)T * H * 2);
  w.pieces_d = w.pieces_gu + weight_gradient_bytes(T, d, 2 * H);      // both products are on their way at a time
  w.bytes = w.pieces_d + weight_gradient_bytes(T, H, d) + 256;
  return w;
}

int gated_check(int32_t T, int32_t d, int32_t H, int32_t act) {
  if (T < 0 || d < 1 || H < 1 || act < GROUTER_ACT_NONE || act > GROUTER_ACT_GELU) return GROUTER_ERR_INVALID_ARG;
  if (d % 8 || H % 8 || !fits_int(T) || !fits_int(d) || !fits_int(2 * (int64_t)H)) return GROUTER_ERR_UNSUPPORTED;
  return GROUTER_OK;
}

// Pieces the contraction of the weight gradient over T tokens is cut into, and their length in 128-deep steps, whole groups of four (a scale
// atom).  Cost in steps of a 256 x 256 tile (0.3 us): rounds of the CTA pairs times what a tile takes or, with dx's product in the same launch,
// the share of a pair in all of it; a sum over pieces takes 10 steps and reads its matrices at 8 TB/s (alone: the backward pass of 16384
// tokens, 1024 x 1024: 99 -> 66 us, 65536 tokens, 256 x 256: 183 -> 52).
struct Fp8Pieces {
  int count, steps;
};
Fp8Pieces fp8_pieces(int T, int K, int N, bool with_dx) {
  const int pairs = current_sms() / 2 > 0 ? current_sms() / 2 : 1, steps = T > 0 ? (T + 127) / 128 : 1, dx_steps = (N + 127) / 128;
  const int64_t tiles = (((int64_t)N + 255) / 256) * (((int64_t)K + 255) / 256), dx_tiles = (((int64_t)T + 255) / 256) * (((int64_t)K + 255) / 256);
  Fp8Pieces best{1, steps};
  float best_cost = 0.f;
  for (int s = 1; s <= 16 && (s == 1 || steps / s >= 8); ++s) {
    const int each = s == 1 ? steps : ((steps + s - 1) / s + 3) / 4 * 4, count = (steps + each - 1) / each;
    float cost = (float)((tiles * count + pairs - 1) / pairs) * fp8_tile_cost(each);
    if (with_dx) {
      const float all = ((float)tiles * count * fp8_tile_cost(each) + (float)dx_tiles * fp8_tile_cost(dx_steps)) / pairs;
      cost = all > cost ? all : cost;
    }
    if (count > 1) cost += 10.f + (float)count * N * K * (4.f / 8e6f / 0.3f);
    if (s == 1 || cost < best_cost) {
      best = {count, each};
      best_cost = cost;
    }
  }
  return best;
}

struct Fp8Workspace {
  size_t rows, row_scales, cols, col_scales, sums, pieces, bytes;
};
// Codes of dy and of its transpose, and the partial sums of its columns.
Fp8Workspace fp8_workspace(int T, int K, int N) {
  Fp8Workspace w{};
  w.row_scales = up256((size_t)T * fp8_pitch(N));
  w.cols = w.row_scales + up256(grouter_fp8_scale_bytes(T, N));
  w.col_scales = w.cols + up256((size_t)N * fp8_pitch(T));
  w.sums = w.col_scales + up256(grouter_fp8_scale_bytes(N, T));
  w.pieces = w.sums + up256(((size_t)T + 127) / 128 * N * 4);
  const int alone = fp8_pieces(T, K, N, false).count, both = fp8_pieces(T, K, N, true).count, count = alone > both ? alone : both;
  w.bytes = w.pieces + (count > 1 ? up256((size_t)count * fp8_piece_rows(N) * K * 4) : 0) + 256;
  return w;
}

// Codes of bf16 activations [T,K], made by the call itself.
struct Fp8Input {
  size_t scales, bytes;
};
Fp8Input fp8_input(int T, int K) {
  Fp8Input w{};
  w.scales = up256((size_t)T * fp8_pitch(K));
  w.bytes = w.scales + up256(grouter_fp8_scale_bytes(T, K));
  return w;
}

int fp8_check(int32_t T, int32_t K, int32_t N) {
  if (T < 0 || K < 1 || N < 1) return GROUTER_ERR_INVALID_ARG;
  if (N % 8 || !fits_int(T) || K > FP8_MAX_COLS || N > FP8_MAX_COLS) return GROUTER_ERR_UNSUPPORTED;
  // the scales' atoms are counted in 32 bits
  const int64_t most = 1 << 30;
  if (((int64_t)T / 128 + 2) * fp8_atoms_across(K) > most || ((int64_t)N / 128 + 2) * fp8_atoms_across(K) > most) return GROUTER_ERR_UNSUPPORTED;
  return GROUTER_OK;
}

// Which of the two kernels is ahead: both sides in microseconds, fitted to measurements over 65 to 4096 tokens and weights of 128 x 128 to
// 8192 x 4096.  Tiles of 256 x 256 (or 128 hidden columns) on CTA pairs: a start and the steps of every round of the pairs.  Few tokens: for
// every round of the SMs a start, the steps of one cut, a meeting of the cluster and, where h is formed, the tokens of a tile.
// Measured (few tokens against tiles): 8 bits 4096 -> 1536, 128 tokens 6.9 and 13.8 us, 1024 tokens 18 and 14; 1024 -> 2816, 512 tokens 7.7 and
// 7.2; 4096 -> 4096, 384 tokens 13 and 15.  Gated in 8 bits d 4096, hidden 1536: 128 tokens 12.7 and 14.5, 512 tokens 16.2 and 15.9;
// d 1024, hidden 2816: 64 tokens 7.5 and 9.5, 128 tokens 11.7 and 7.8.  In bf16 the same: 128 tokens 17 and 26.5, 1024 tokens 34 and 26;
// 64 tokens 6.5 and 9.4, 256 tokens 11.0 and 9.7.
// Up to 64 tokens it always is, by more the larger the weight (whole gated block, d 2048, hidden 8192: 8 tokens 23 and 65 us, 64 tokens 30 and 33;
// d 8192, hidden 8192: 66 and 90, 73 and 82; 8 bits 4096 -> 22016: 13 and 39, 15 and 17).
inline int rounds(int64_t tiles, int places) { return (int)((tiles + places - 1) / (places > 0 ? places : 1)); }
inline int log2_of(int s) { return s >= 8 ? 3 : s >= 4 ? 2 : s >= 2 ? 1 : 0; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int token_tile(int T) { return T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128; }

// Whether the kernel for few tokens is ahead, in `splits` cuts.
bool fp8_few(const Fp8Gemm& g, int& splits) {
  const bool glu = g.B1.codes != nullptr;
  const int sms = current_sms();
  splits = fp8_small_splits(g.M, g.N, g.K, glu);
  const int64_t steps = cdiv(g.K, 128), ctas = cdiv(g.N, 128) * cdiv(g.M, 128) * splits;
  const int tile_rounds = rounds(cdiv(g.M, 256) * cdiv(g.N, glu ? 128 : 256), sms / 2);
  const float tiles = (glu ? 4.9f + 0.31f * steps * tile_rounds : 4.4f + 0.285f * steps * tile_rounds);
  const float small = glu ? rounds(ctas, sms) * (2.9f + 0.045f * token_tile(g.M) + 0.45f * cdiv(steps, splits) + 0.8f * log2_of(splits))
                          : rounds(ctas, 2 * sms) * (3.f + 0.48f * cdiv(steps, splits) + log2_of(splits));
  const bool fits = cdiv(g.M, 128) <= 65535;      // its grid has the token tiles in y
  return !g.out_f32 && fits && (g.M <= 64 || small < tiles);
}
// A as codes, or (g.x) as bf16, which a kernel of its own puts into the place that g.A names unless the product can do it on the way.
cudaError_t fp8_product(Fp8Gemm g, cudaStream_t st) {
  int splits;
  const bool few = fp8_few(g, splits);
  if (g.x && !(few && g.M <= 16 && g.K % 8 == 0 && g.ldx % 8 == 0 && aligned_to(g.x, 16))) {
    if (const cudaError_t e = launch_quantize(g.x, g.ldx, GROUTER_BF16, g.M, g.K, false, const_cast<void*>(g.A.codes), const_cast<void*>(g.A.scales),
                                              nullptr, nullptr, nullptr, st))
      return e;
    g.x = nullptr;
  }
  return few ? launch_fp8_small(g, splits, st) : launch_fp8_gemm(g, st);
}
cudaError_t gated_product(const GatedGemm& g, cudaStream_t st) {
  const int sms = current_sms(), splits = gated_small_splits(g.T, g.H, g.K);
  const int64_t steps = cdiv(g.K, 64), ctas = cdiv(2 * (int64_t)g.H, 128) * cdiv(g.T, 128) * splits;
  const float tiles = 5.f + 0.3f * steps * rounds(cdiv(g.T, 256) * cdiv(g.H, 128), sms / 2);
  const float small = rounds(ctas, 2 * sms) * (2.f + 0.03f * token_tile(g.T) + 0.5f * cdiv(steps, splits));
  return cdiv(g.T, 128) <= 65535 && (g.T <= 64 || small < tiles) ? launch_gated_small(g, splits, st) : launch_gated_gemm(g, st);
}

}  // namespace
}  // namespace grouter

using namespace grouter;

extern "C" {

int grouter_gated_ffn_fwd(const void* x, const void* W_gu, const void* W_d, const void* residual, int32_t T, int32_t d, int32_t H, int32_t act,
                          void* h, void* y, void* pre, int32_t* status, void* stream) {
  if (const int e = gated_check(T, d, H, act)) return e;
  if (!W_gu || !W_d || !status || (T > 0 && (!x || !h || !y))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(x, 16) || !aligned_to(W_gu, 16) || !aligned_to(W_d, 16) || !aligned_to(residual, 16) || !aligned_to(h, 16) || !aligned_to(y, 16) ||
      !aligned_to(pre, 16) || !aligned_to(status, 4))
    return GROUTER_ERR_MISALIGNED;
  if (T == 0) return GROUTER_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  GatedGemm g{};
  g.A = x; g.W = W_gu; g.pre = pre; g.h = h; g.T = T; g.K = d; g.H = H; g.act = act; g.status = status;
  if (gated_product(g, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  LinearGemm l{};
  l.A = h; l.B = W_d; l.residual = residual; l.C = y; l.M = T; l.N = d; l.K = H; l.act = GROUTER_ACT_NONE; l.status = status;
  return launch_product(l, st) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

size_t grouter_gated_ffn_bwd_workspace_bytes(int32_t T, int32_t d, int32_t H) {
  if (gated_check(T, d, H, GROUTER_ACT_NONE) != GROUTER_OK) return 0;
  return gated_workspace(T, d, H).bytes;
}

int grouter_gated_ffn_bwd(const void* dy, const void* x, const void* W_gu, const void* W_d, const void* pre, int32_t T, int32_t d, int32_t H,
                          int32_t act, void* dx, void* dW_gu, void* dW_d, int32_t dW_dtype, void* workspace, int32_t* status, void* stream) {
  if (const int e = gated_check(T, d, H, act)) return e;
  if (!status || (!dx && !dW_gu && !dW_d) || (dW_dtype != GROUTER_BF16 && dW_dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  if (T > 0 && (!dy || !W_d || !pre || !workspace || (dx && !W_gu) || (dW_gu && !x))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(dy, 16) || !aligned_to(x, 16) || !aligned_to(W_gu, 16) || !aligned_to(W_d, 16) || !aligned_to(pre, 16) || !aligned_to(dx, 16) ||
      !aligned_to(dW_gu, 16) || !aligned_to(dW_d, 16) || !aligned_to(workspace, 256) || !aligned_to(status, 4))
    return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {           // sums over no tokens
    const size_t el = dW_dtype == GROUTER_F32 ? 4 : 2;
    if (dW_gu && cudaMemsetAsync(dW_gu, 0, (size_t)2 * H * d * el, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    if (dW_d && cudaMemsetAsync(dW_d, 0, (size_t)d * H * el, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    return GROUTER_OK;
  }
  const GatedWorkspace w = gated_workspace(T, d, H);
  char* ws = static_cast<char*>(workspace);
  GatedGemm g{};
  g.A = dy; g.W = W_d; g.pre = const_cast<void*>(pre); g.dpre = ws + w.dp; g.h = ws + w.h; g.T = T; g.K = d; g.H = H; g.act = act;
  g.backward = true; g.status = status;
  if (launch_gated_gemm(g, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  if (dx) {
    LinearGemm l{};
    l.A = ws + w.dp; l.B = W_gu; l.b_mn = 1; l.C = dx; l.M = T; l.N = d; l.K = 2 * H; l.act = GROUTER_ACT_NONE; l.status = status;
    if (launch_product(l, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  }
  // The three products read what the first kernel wrote and nothing of one another: each works beside the end of the one before it, whose
  // last round leaves pairs of SMs idle (4095 x 1024, hidden 2816: 64, 88 and 44 tiles for 74 pairs).  The first of them, dx's where it is
  // wanted, waits for the first kernel at its start; the others rely on that one's wait, dW_d's on the far side of dW_gu's, which does not wait
  // before it lets dW_d's start (launch_dependent, vec.cuh).
  bool beside = dx != nullptr;
  if (dW_gu) {
    if (launch_weight_product(ws + w.dp, x, T, d, 2 * H, dW_gu, dW_dtype, ws + w.pieces_gu, status, beside, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    beside = true;
  }
  if (dW_d && launch_weight_product(dy, ws + w.h, T, H, d, dW_d, dW_dtype, ws + w.pieces_d, status, beside, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  if (dW_gu && launch_weight_sum(T, d, 2 * H, dW_gu, dW_dtype, ws + w.pieces_gu, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  if (dW_d && launch_weight_sum(T, H, d, dW_d, dW_dtype, ws + w.pieces_d, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  return GROUTER_OK;
}

size_t grouter_linear_fp8_fwd_workspace_bytes(int32_t T, int32_t K) {
  return fp8_check(T, K, 8) != GROUTER_OK ? 0 : fp8_input(T, K).bytes;
}

int grouter_linear_fp8_fwd(const void* x, const void* x_scales, int64_t ldx, const void* W, const void* W_scales, const void* bias,
                           const void* residual, int32_t T, int32_t K, int32_t N, void* y, void* workspace, int32_t* status, void* stream) {
  if (const int e = fp8_check(T, K, N)) return e;
  if (!W || !W_scales || !status || (T > 0 && (!x || !y || (!x_scales && (!workspace || ldx < K))))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(x, x_scales ? 16 : 2) || !aligned_to(x_scales, 16) || !aligned_to(W, 16) || !aligned_to(W_scales, 16) || !aligned_to(bias, 16) ||
      !aligned_to(residual, 16) || !aligned_to(y, 16) || !aligned_to(workspace, 256) || !aligned_to(status, 4))
    return GROUTER_ERR_MISALIGNED;
  if (T == 0) return GROUTER_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Fp8Gemm g{};
  g.A = {x, x_scales};
  if (!x_scales) {
    char* ws = static_cast<char*>(workspace);
    g.A = {ws, ws + fp8_input(T, K).scales};
    g.x = x;
    g.ldx = ldx;
  }
  g.B = {W, W_scales}; g.bias = bias; g.residual = residual; g.C = y; g.M = T; g.N = N; g.K = K; g.status = status;
  return fp8_product(g, st) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

size_t grouter_linear_fp8_bwd_workspace_bytes(int32_t T, int32_t K, int32_t N) {
  if (fp8_check(T, K, N) != GROUTER_OK || K % 8 || T > FP8_MAX_COLS) return 0;
  return fp8_workspace(T, K, N).bytes;
}

int grouter_linear_fp8_bwd(const void* dy, const void* xt, const void* xt_scales, const void* Wt, const void* Wt_scales, int32_t T, int32_t K, int32_t N,
                           void* dx, void* dW, int32_t dW_dtype, float* db, void* workspace, int32_t* status, void* stream) {
  if (const int e = fp8_check(T, K, N)) return e;
  if (K % 8 || T > FP8_MAX_COLS) return GROUTER_ERR_UNSUPPORTED;
  if (!status || (!dx && !dW && !db) || (dW_dtype != GROUTER_BF16 && dW_dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  if (T > 0 && (!dy || !workspace || (dx && (!Wt || !Wt_scales)) || (dW && (!xt || !xt_scales)))) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(dy, 16) || !aligned_to(xt, 16) || !aligned_to(xt_scales, 16) || !aligned_to(Wt, 16) || !aligned_to(Wt_scales, 16) || !aligned_to(dx, 16) ||
      !aligned_to(dW, 16) || !aligned_to(db, 4) || !aligned_to(workspace, 256) || !aligned_to(status, 4))
    return GROUTER_ERR_MISALIGNED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {           // sums over no tokens
    if (dW && cudaMemsetAsync(dW, 0, (size_t)N * K * (dW_dtype == GROUTER_F32 ? 4 : 2), st) != cudaSuccess) return GROUTER_ERR_CUDA;
    if (db && cudaMemsetAsync(db, 0, (size_t)N * 4, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    return GROUTER_OK;
  }
  const Fp8Workspace w = fp8_workspace(T, K, N);
  char* ws = static_cast<char*>(workspace);
  // the sums are taken on the way to the transposed codes, which a bias alone does not need
  const int tiles = (T + 127) / 128;
  float* sums = db ? (tiles == 1 ? db : reinterpret_cast<float*>(ws + w.sums)) : nullptr;
  const bool columns = dW || db;
  if (launch_quantize(dy, N, GROUTER_BF16, T, N, false, dx ? ws : nullptr, ws + w.row_scales, columns ? ws + w.cols : nullptr, ws + w.col_scales, sums,
                      st) != cudaSuccess)
    return GROUTER_ERR_CUDA;
  if (db && tiles > 1 && launch_sum_rows(sums, tiles, N, db, N, nullptr, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  Fp8Gemm to_x{}, to_w{};
  to_x.A = {ws, ws + w.row_scales}; to_x.B = {Wt, Wt_scales}; to_x.C = dx; to_x.M = T; to_x.N = K; to_x.K = N; to_x.status = status;
  to_w.A = {ws + w.cols, ws + w.col_scales}; to_w.B = {xt, xt_scales}; to_w.C = dW; to_w.M = N; to_w.N = K; to_w.K = T; to_w.status = status;
  to_w.out_f32 = dW_dtype == GROUTER_F32;
  // Both on tiles go in one launch: the gradient of a weight has few of them, of long contractions, and leaves pairs of SMs without one, which
  // work on dx's meanwhile (16384 tokens, 1408 x 2048: 48 tiles of 128 steps and 512 of 11 on 74 pairs: the backward pass 105 us, one after the other 112).
  int splits;
  const bool together = dx && dW && !fp8_few(to_x, splits);
  const Fp8Pieces pieces = fp8_pieces(T, K, N, together);
  if (pieces.count > 1) {
    to_w.C = ws + w.pieces;
    to_w.out_f32 = 1;
    to_w.pieces = pieces.count;
    to_w.piece_steps = pieces.steps;
  }
  if (together) {
    const bool w_first = pieces.steps >= cdiv(N, 128);
    if (launch_fp8_gemms(w_first ? to_w : to_x, w_first ? to_x : to_w, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  } else {
    if (dx && fp8_product(to_x, st) != cudaSuccess) return GROUTER_ERR_CUDA;
    to_w.waits_at_end = dx != nullptr;       // of dx's product, which waits at its start for the codes (and sums of db), it needs nothing
    if (dW && launch_fp8_gemm(to_w, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  }
  if (dW && pieces.count > 1 &&
      launch_sum_pieces(ws + w.pieces, pieces.count, (int64_t)N * K, (int64_t)fp8_piece_rows(N) * K, dW, dW_dtype, st) != cudaSuccess)
    return GROUTER_ERR_CUDA;
  return GROUTER_OK;
}

size_t grouter_gated_ffn_fp8_fwd_workspace_bytes(int32_t T, int32_t d, int32_t H) {
  if (gated_check(T, d, H, GROUTER_ACT_NONE) != GROUTER_OK || fp8_check(T, d, H) != GROUTER_OK || fp8_check(T, H, d) != GROUTER_OK) return 0;
  return fp8_input(T, d).bytes + fp8_input(T, H).bytes;
}

int grouter_gated_ffn_fp8_fwd(const void* x, const void* x_scales, int64_t ldx, const void* W_g, const void* W_g_scales, const void* W_u,
                              const void* W_u_scales, const void* W_d, const void* W_d_scales, const void* residual, int32_t T, int32_t d, int32_t H,
                              int32_t act, void* y, void* workspace, int32_t* status, void* stream) {
  if (const int e = gated_check(T, d, H, act)) return e;
  if (fp8_check(T, d, H) || fp8_check(T, H, d)) return GROUTER_ERR_UNSUPPORTED;
  if (!W_g || !W_g_scales || !W_u || !W_u_scales || !W_d || !W_d_scales || !status || (T > 0 && (!x || !y || !workspace || (!x_scales && ldx < d))))
    return GROUTER_ERR_INVALID_ARG;
  for (const void* q : {x_scales ? x : nullptr, x_scales, W_g, W_g_scales, W_u, W_u_scales, W_d, W_d_scales, residual, (const void*)y})
    if (!aligned_to(q, 16)) return GROUTER_ERR_MISALIGNED;
  if (!aligned_to(x, 2) || !aligned_to(workspace, 256) || !aligned_to(status, 4)) return GROUTER_ERR_MISALIGNED;
  if (T == 0) return GROUTER_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char *ws = static_cast<char*>(workspace), *h = ws + fp8_input(T, d).bytes, *h_scales = h + fp8_input(T, H).scales;
  Fp8Gemm g{};
  g.A = {x, x_scales};
  if (!x_scales) {
    g.A = {ws, ws + fp8_input(T, d).scales};
    g.x = x;
    g.ldx = ldx;
  }
  g.B = {W_g, W_g_scales}; g.B1 = {W_u, W_u_scales}; g.C = h; g.out_scales = h_scales; g.M = T; g.N = H; g.K = d; g.act = act;
  g.status = status;
  if (fp8_product(g, st) != cudaSuccess) return GROUTER_ERR_CUDA;
  Fp8Gemm l{};
  l.A = {h, h_scales}; l.B = {W_d, W_d_scales}; l.residual = residual; l.C = y; l.M = T; l.N = d; l.K = H; l.status = status;
  return fp8_product(l, st) == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
