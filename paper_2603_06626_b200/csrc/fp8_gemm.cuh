// Products of matrices in 8 bits, as the operators launch them.
#pragma once
#include "common.cuh"

namespace grouter {

struct Fp8Operand {
  const void *codes, *scales;             // [rows, fp8_pitch(cols)], packed scales (fp8.cuh)
};
// C [M,N] = A B^T + bias + residual, bf16 or f32; with B1: act(A B^T) (A B1^T) as codes C and out_scales.
struct Fp8Gemm {
  Fp8Operand A, B, B1;
  const void* x;                          // A as bf16, row t at x + t * ldx, instead of codes (launch_fp8_small, up to 16 rows); else null
  int64_t ldx;
  const void *bias, *residual;            // bf16 or null
  void *C, *out_scales;
  int M, N, K, act, out_f32;
  int32_t* status;
  int pieces, piece_steps;                // with out_f32, over 1: C [pieces][fp8_piece_rows(M)][N] of partial products over piece_steps 128-deep steps each
  bool waits_at_end;                      // launch_fp8_gemm: works beside the end of the kernels before it, back to the last that waited at its start (vec.cuh)
};
cudaError_t launch_fp8_gemm(const Fp8Gemm& g, cudaStream_t st);
// Two products that need nothing of one another, bf16 or f32 out, in one launch; a is the one with the longer contraction (or pieces).
cudaError_t launch_fp8_gemms(const Fp8Gemm& a, const Fp8Gemm& b, cudaStream_t st);
// What a tile of so many 128-deep steps takes, in steps: four of them pass between two tiles.
inline int fp8_tile_cost(int steps) { return steps + 4; }
inline int fp8_piece_rows(int M) { return (M + 31) / 32 * 32; }
// The same for few rows of A (tokens), bf16 or codes out: the contraction cut over a cluster of `splits` CTAs (fp8_small_splits).
int fp8_small_splits(int T, int N, int K, bool glu);
cudaError_t launch_fp8_small(const Fp8Gemm& g, int splits, cudaStream_t st);
// Tensor maps of a matrix's codes (tiles of 128 columns x box_rows) and of its scales (one 512-byte atom).
bool make_fp8_maps(CUtensorMap* codes, CUtensorMap* scales, const Fp8Operand& x, int rows, int cols, uint32_t box_rows);
// Codes of the rows of x and, with codes_t, of its columns; column_sums: with codes_t, f32 [ceil(rows / 128), cols] of the tiles' sums.
cudaError_t launch_quantize(const void* x, int64_t ldx, int dtype, int rows, int cols, bool square, void* codes, void* scales, void* codes_t,
                            void* scales_t, float* column_sums, cudaStream_t st);

}  // namespace grouter
