// Matrices into 8 bits and back (the format is in fp8.cuh): codes of the rows, of the transposed matrix, or both from one reading.
//
// Bound by HBM (2 bytes in and one out an element, two out with the transposed codes) as long as an element costs no more than the 17
// (rows) or 22 (both) instruction slots that its bytes leave it; so a lane takes sixteen neighbours, over which addresses, exponent and
// shuffles are spread.  bf16 stays in pairs: magnitudes are compared two to an instruction as 16-bit integers (their order is that of the
// numbers), infinities and NaN are looked for in the maximum only, and two elements are scaled and converted by one instruction each.
// Measured: 32768 x 4096 bf16 to codes of the rows 60 us (6.7 TB/s), of both forms 93 (5.8), back to bf16 61; f32 both forms 201.
// Squares (weights), rows and both forms: 4096 x 4096 10 and 15 us, 22016 x 4096 42 and 64.  Rows that are not 16-byte aligned (an odd stride or
// width) come element by element: 32768 x 4096 145 us for the rows, 166 for both forms; a stride of 4104 keeps the wide accesses (61, 104).
//   Rows alone: eight lanes hold a block of 128, a warp four blocks (whose scales are one word) of two rows.
//   Squares or transposed codes: a CTA takes a tile of 128 x 128, which is a block of every row, a block of every column and a whole
//     square.  For the transposed codes it waits in shared memory and is read by columns: a lane takes sixteen neighbouring rows of a word's
//     columns (two of bf16), eight lanes hold a column (with eight rows and sixteen lanes 32768 x 4096 121 us, f32 316); words are permuted so
//     that these reads meet no conflicts.
#include "fp8.cuh"
#include "fp8_gemm.cuh"

namespace grouter {

constexpr int QT = 128;                   // the tile's sides
constexpr int Q_THREADS = 256;

struct QuantParams {
  const void* x;
  int64_t ldx;
  int rows, cols;
  uint8_t *codes, *scales;                // of the rows [rows, pitch(cols)], or null
  uint8_t *codes_t, *scales_t;            // of the columns [cols, pitch(rows)], or null
  float* sums;                            // with codes_t: [tile rows, cols] sums of a tile's columns, or null
  int64_t tiles_c;
};

// Sixteen elements of a row from column c on; zeros outside the matrix.
template <typename T, bool VEC>
__device__ __forceinline__ void load_lane(const T* at, int c, int cols, bool row_there, uint32_t (&w)[q_words<T>()]) {
  constexpr int VE = vec16<T>();
#pragma unroll
  for (int i = 0; i < Q_LANE / VE; ++i) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (VEC) {
      if (row_there && c + i * VE < cols) v = ld_stream16(at + i * VE);
    } else {
      T* e = reinterpret_cast<T*>(&v);
#pragma unroll
      for (int k = 0; k < VE; ++k)
        if (row_there && c + i * VE + k < cols) e[k] = at[i * VE + k];
    }
    w[4 * i] = v.x;
    w[4 * i + 1] = v.y;
    w[4 * i + 2] = v.z;
    w[4 * i + 3] = v.w;
  }
}
// Where a lane of the kernels over rows works: QR_ROWS rows from r0 on, 512 columns (an atom's) from `chunk` on with the other lanes of its warp;
// where rows are no longer than 256 or 128 elements, half a warp or a quarter does (200000 x 96 to codes 29.3 -> 10.0 us).  A block's eight warps
// are 2^across_log2 beside one another, the others below.
constexpr int QR_ROWS = 2;                // one, two, four: 8 x 4096 to codes 1.3, 1.5, 2.0 us, 65536 x 256 8.2, 7.8, 8.3, 32768 x 4096 in f32 108, 108, 114
struct RowsShape {
  int across_log2, lanes_log2;
};
struct RowsPlace {
  int warp_r0, r0, chunk, lane;           // lane: within those that share rows
};
__device__ __forceinline__ RowsPlace rows_place(RowsShape shape) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, across = 1 << shape.across_log2;
  const int w0 = (((int)blockIdx.x * ((Q_THREADS / 32) >> shape.across_log2) + (warp >> shape.across_log2)) << (5 - shape.lanes_log2)) * QR_ROWS;
  return {w0, w0 + (lane >> shape.lanes_log2) * QR_ROWS, (int)blockIdx.y * across + (warp & (across - 1)), lane & ((1 << shape.lanes_log2) - 1)};
}

// Codes of the rows alone.
template <typename T, bool VEC>
__global__ void __launch_bounds__(Q_THREADS) quantize_rows_kernel(const QuantParams p, RowsShape shape) {
  const RowsPlace at = rows_place(shape);
  const int c = at.chunk * 4 * QT + at.lane * Q_LANE;
  const int pitch = (int)fp8_pitch(p.cols), across = (int)fp8_atoms_across(p.cols);
  after_previous_kernel();
  let_next_kernel_start();
  if (at.warp_r0 >= p.rows || at.chunk >= across) return;        // whole warps
  const T* x = static_cast<const T*>(p.x) + at.r0 * p.ldx + c;
  uint32_t w[QR_ROWS][q_words<T>()];
#pragma unroll
  for (int n = 0; n < QR_ROWS; ++n) load_lane<T, VEC>(x + n * p.ldx, c, p.cols, at.r0 + n < p.rows, w[n]);
  uint8_t* to = p.codes + (int64_t)at.r0 * pitch + c;
  uint8_t* scale = p.scales + fp8_scale_at(at.r0, 4 * at.chunk + at.lane / Q_LANES, across);      // of the rows below: 16 bytes on each
  const bool here = c < pitch, says = here && (at.lane & (Q_LANES - 1)) == 0;
  bool inf;
  uint32_t e[QR_ROWS];
  block_exponents<T>(w, e, inf);
#pragma unroll
  for (int n = 0; n < QR_ROWS; ++n) {
    const float2 inv = both(fp8_inverse(e[n]));
    const uint4 q = inf ? lane_codes<T, true>(w[n], inv) : lane_codes<T, false>(w[n], inv);
    if (at.r0 + n < p.rows) {
      if (here) *reinterpret_cast<uint4*>(to + (int64_t)n * pitch) = q;
      if (says) scale[16 * n] = (uint8_t)e[n];
    }
  }
}

template <typename T, bool VEC, bool SQUARE>
__global__ void __launch_bounds__(Q_THREADS, sizeof(T) == 2 ? 4 : 2) quantize_tile_kernel(const QuantParams p) {
  constexpr int W = q_words<T>(), STEP = Q_THREADS / Q_LANES, NR = QT / STEP;        // rows a block at a time, times
  constexpr int WORDS = QT * (int)sizeof(T) / 4;                                     // of a tile row
  extern __shared__ __align__(16) uint32_t s_tile[];   // [QT][WORDS], with transposed codes; word w of row r at place(w, r)
  __shared__ uint32_t s_top[2][Q_THREADS / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = threadIdx.x / Q_LANES, at = threadIdx.x % Q_LANES;
  const int tiles_c = (int)p.tiles_c, tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
  const int r0 = tr * QT, c0 = tc * QT, c = c0 + at * Q_LANE;
  after_previous_kernel();
  let_next_kernel_start();
  // four words at a time stay together, and no two of a warp's go to the same banks, neither when rows are written nor when columns are read
  auto place = [](int w, int r16) { return w ^ ((r16 ^ (w >> 5 & 3)) << 2); };
  uint32_t v[NR / 2][2][W];
  const T* x = static_cast<const T*>(p.x) + (int64_t)(r0 + sub) * p.ldx + c;
#pragma unroll
  for (int n = 0; n < NR; ++n) load_lane<T, VEC>(x + n * STEP * p.ldx, c, p.cols, r0 + n * STEP + sub < p.rows, v[n / 2][n & 1]);
  uint32_t square = 0;
  bool square_inf = false;
  if (SQUARE) {
    auto block_top = [&](uint32_t t, int which) {
      t = lanes_top_bits<32>(t);
      if (lane == 0) s_top[which][warp] = t;
      __syncthreads();
      t = s_top[which][0];
#pragma unroll
      for (int w = 1; w < Q_THREADS / 32; ++w) t = max(t, s_top[which][w]);
      return t;
    };
#pragma unroll
    for (int n = 0; n < NR; ++n) square = max(square, lane_top<T>(v[n / 2][n & 1]));
    square = block_top(square, 0);
    square_inf = bits_not_finite(square);
    if (square_inf) {                     // the whole block alike
      square = 0;
#pragma unroll
      for (int n = 0; n < NR; ++n) square = max(square, lane_top_finite<T>(v[n / 2][n & 1]));
      square = block_top(square, 1);
    }
  }
  if (p.codes_t) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = n * STEP + sub;
      uint32_t* row = s_tile + r * WORDS;
      const uint32_t* w = v[n / 2][n & 1];
#pragma unroll
      for (int i = 0; i < W; i += 4) *reinterpret_cast<uint4*>(row + place(at * W + i, r >> 4)) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
  }
  if (p.codes) {
    const int pitch = (int)fp8_pitch(p.cols);
    const int64_t across = fp8_atoms_across(p.cols);
    uint8_t* to = p.codes + (int64_t)(r0 + sub) * pitch + c;
    uint8_t* scale = p.scales + (tr * across + (tc >> 2)) * FP8_ATOM + (tc & 3);
    const bool here = c < pitch;
#pragma unroll
    for (int m = 0; m < NR / 2; ++m) {
      bool inf = square_inf;
      uint32_t e[2];
      if (SQUARE) e[0] = e[1] = fp8_exponent(__uint_as_float(square));
      else block_exponents<T>(v[m], e, inf);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = (2 * m + k) * STEP + sub;
        const float2 inv = both(fp8_inverse(e[k]));
        const uint4 q = inf ? lane_codes<T, true>(v[m][k], inv) : lane_codes<T, false>(v[m][k], inv);
        if (r0 + r < p.rows && here) {
          *reinterpret_cast<uint4*>(to + (int64_t)((2 * m + k) * STEP) * pitch) = q;
          if (at == 0) scale[(r & 31) * 16 + (r >> 5) * 4] = (uint8_t)e[k];
        }
      }
    }
  }
  if (p.codes_t) {
    __syncthreads();
    constexpr int CPW = 4 / (int)sizeof(T);             // columns of a word
    constexpr int UNROLL = sizeof(T) == 2 ? 2 : 1;      // f32: four times no faster
    const int64_t pitch = fp8_pitch(p.rows);
    const int lr = lane & 7, side = lane >> 3;          // rows 16 lr .. 16 lr + 15 of one of four neighbouring words
    const bool here = r0 + 16 * lr < pitch;
    const uint32_t* from = s_tile + 16 * lr * WORDS;
    uint8_t* to = p.codes_t + c0 * pitch + r0 + 16 * lr;
    uint8_t* scale = p.scales_t + (tc * fp8_atoms_across(p.rows) + (tr >> 2)) * FP8_ATOM + (tr & 3);
#pragma unroll UNROLL
    for (int w4 = warp; w4 < WORDS / 4; w4 += Q_THREADS / 32) {
      const int word = 4 * w4 + side;
      uint32_t q[16], tops = 0;                         // tops: of the word's columns
#pragma unroll
      for (int i = 0; i < 16; ++i) q[i] = from[i * WORDS + place(word, lr)];
      bool inf = square_inf;
      if (!SQUARE) {
#pragma unroll
        for (int i = 0; i < 16; ++i) tops = word_top<T>(tops, q[i]);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) tops = word_top<T>(tops, __shfl_xor_sync(0xffffffffu, tops, o));
        inf = __any_sync(0xffffffffu, bits_not_finite(top_of_word<T>(tops)));
        if (inf) {
          tops = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) tops = word_top_finite<T>(tops, q[i]);
#pragma unroll
          for (int o = 4; o > 0; o >>= 1) tops = word_top<T>(tops, __shfl_xor_sync(0xffffffffu, tops, o));
        }
      }
#pragma unroll
      for (int j = 0; j < CPW; ++j) {
        auto half = [&](uint32_t w) { return sizeof(T) == 4 ? w : j == 0 ? w << 16 : w & 0xffff0000u; };
        float f[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(half(q[i]));
        const uint32_t e = fp8_exponent(__uint_as_float(SQUARE ? square : half(tops)));
        const float inv = fp8_inverse(e);
        const int col = word * CPW + j;                 // within the tile
        const bool column = c0 + col < p.cols;
        if (p.sums) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 16; i += 4) sum += (f[i] + f[i + 1]) + (f[i + 2] + f[i + 3]);
          sum = lanes_sum<8>(sum);
          if (lr == 0 && column) p.sums[(int64_t)tr * p.cols + c0 + col] = sum;
        }
        uint32_t codes[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) codes[i] = inf ? fp8_quad<true>(f + 4 * i, inv) : fp8_quad<false>(f + 4 * i, inv);
        if (column && here) {
          *reinterpret_cast<uint4*>(to + col * pitch) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
          if (lr == 0) scale[(col & 31) * 16 + (col >> 5) * 4] = (uint8_t)e;
        }
      }
    }
  }
}

// Rows of 512 columns a warp, as quantize_rows_kernel, but a lane has as many neighbouring codes as fill 16 bytes of the output: a warp's
// stores then fill whole lines (with sixteen codes a lane every other 16 bytes: 32768 x 4096 to bf16 71 us, so 61).  The four scales of a
// row are one word.  Where the output's rows are not 16-byte aligned its elements are stored one by one.
template <typename T>
__global__ void __launch_bounds__(Q_THREADS) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int cols,
                                                               int64_t ldy, bool vec, RowsShape shape, T* __restrict__ y) {
  constexpr int VE = vec16<T>(), WORDS = VE / 4, NJ = 4 * QT / (32 * VE);
  const RowsPlace at = rows_place(shape);
  const int span = VE << shape.lanes_log2, c = at.chunk * 4 * QT + at.lane * VE;
  const int pitch = (int)fp8_pitch(cols), across = (int)fp8_atoms_across(cols);
  after_previous_kernel();
  let_next_kernel_start();
  if (at.r0 >= rows || at.chunk >= across) return;
  const uint8_t* from = codes + (int64_t)at.r0 * pitch + c;
  const uint8_t* scale = scales + fp8_scale_at(at.r0, 4 * at.chunk, across);
  uint32_t q[QR_ROWS][NJ][WORDS], four[QR_ROWS];
#pragma unroll
  for (int n = 0; n < QR_ROWS; ++n) {
    if (at.r0 + n >= rows) break;
    four[n] = __ldg(reinterpret_cast<const uint32_t*>(scale + 16 * n));
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (c + j * span >= pitch) break;
      const uint32_t* w = reinterpret_cast<const uint32_t*>(from + (int64_t)n * pitch + j * span);
      if constexpr (WORDS == 2) {
        const uint2 two = __ldcs(reinterpret_cast<const uint2*>(w));
        q[n][j][0] = two.x;
        q[n][j][1] = two.y;
      } else {
        q[n][j][0] = __ldcs(w);
      }
    }
  }
  T* to = y + at.r0 * ldy + c;
#pragma unroll
  for (int n = 0; n < QR_ROWS; ++n) {
    if (at.r0 + n >= rows) break;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int first = c + j * span;
      if (first >= cols) break;
      const int block = (j * span + at.lane * VE) / QT;
      const float s = fp8_scale(four[n] >> (8 * block) & 0xffu);
      float f[VE];
#pragma unroll
      for (int i = 0; i < VE; i += 2) {
        const float2 t = mul2(fp8_values(q[n][j][i / 4] >> (8 * (i & 2))), both(s));
        f[i] = t.x;
        f[i + 1] = t.y;
      }
      if (vec && first + VE <= cols) {
        st_pack<T, VE>(to + n * ldy + j * span, f);
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (first + i < cols) to[n * ldy + j * span + i] = from_f32<T>(f[i]);
      }
    }
  }
}

namespace {

struct RowsGrid {
  dim3 grid;
  RowsShape shape;
};
RowsGrid rows_grid(int rows, int cols) {
  const int chunks = (int)fp8_atoms_across(cols), lanes = cols <= QT ? 3 : cols <= 2 * QT ? 4 : 5;
  int l = 0;
  while (l < 3 && (1 << l) < chunks) ++l;
  const int64_t block_rows = (((Q_THREADS / 32) >> l) << (5 - lanes)) * QR_ROWS;
  return {dim3((unsigned)((rows + block_rows - 1) / block_rows), (unsigned)((chunks + (1 << l) - 1) >> l)), {l, lanes}};
}

template <typename T, bool VEC, bool SQUARE>
cudaError_t tile_launch(const QuantParams& p, cudaStream_t st) {
  constexpr int smem = QT * QT * (int)sizeof(T);
  auto kern = quantize_tile_kernel<T, VEC, SQUARE>;
  static bool configured[64] = {};        // the opt-in to more than 48 KB of dynamic shared memory, once per device
  int dev = 0;
  cudaGetDevice(&dev);
  if (smem > 48 * 1024 && (dev < 0 || dev >= 64 || !configured[dev])) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  const int64_t blocks = ((int64_t)p.rows + QT - 1) / QT * p.tiles_c;
  return launch_dependent(kern, dim3((unsigned)blocks), dim3(Q_THREADS), p.codes_t ? smem : 0, st, p);
}

template <typename T, bool VEC>
cudaError_t quantize_launch(const QuantParams& p, bool square, cudaStream_t st) {
  if (square) return tile_launch<T, VEC, true>(p, st);
  if (p.codes_t) return tile_launch<T, VEC, false>(p, st);
  const RowsGrid g = rows_grid(p.rows, p.cols);
  return launch_dependent(quantize_rows_kernel<T, VEC>, g.grid, dim3(Q_THREADS), 0, st, p, g.shape);
}

}  // namespace

cudaError_t launch_quantize(const void* x, int64_t ldx, int dtype, int rows, int cols, bool square, void* codes, void* scales, void* codes_t,
                            void* scales_t, float* column_sums, cudaStream_t st) {
  QuantParams p{};
  p.x = x;
  p.ldx = ldx;
  p.rows = rows;
  p.cols = cols;
  p.codes = static_cast<uint8_t*>(codes);
  p.scales = static_cast<uint8_t*>(scales);
  p.codes_t = static_cast<uint8_t*>(codes_t);
  p.scales_t = static_cast<uint8_t*>(scales_t);
  p.sums = column_sums;
  p.tiles_c = ((int64_t)cols + QT - 1) / QT;
  const int ve = dtype == GROUTER_F32 ? 4 : 8;
  const bool vec = aligned_to(x, 16) && ldx % ve == 0 && cols % ve == 0;
  if (dtype == GROUTER_F32) return vec ? quantize_launch<float, true>(p, square, st) : quantize_launch<float, false>(p, square, st);
  return vec ? quantize_launch<__nv_bfloat16, true>(p, square, st) : quantize_launch<__nv_bfloat16, false>(p, square, st);
}

}  // namespace grouter

using namespace grouter;

extern "C" {

size_t grouter_fp8_pitch(int32_t cols) { return cols < 0 ? 0 : (size_t)fp8_pitch(cols); }
size_t grouter_fp8_scale_bytes(int32_t rows, int32_t cols) {
  return rows < 0 || cols < 0 ? 0 : ((size_t)rows + 127) / 128 * (size_t)fp8_atoms_across(cols) * FP8_ATOM;
}

int grouter_quantize_fp8(const void* x, int64_t ldx, int32_t dtype, int32_t rows, int32_t cols, int32_t square, void* codes, void* scales,
                         void* codes_t, void* scales_t, void* stream) {
  if (rows < 0 || cols < 0 || ldx < cols || (dtype != GROUTER_BF16 && dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  if (rows > INT32_MAX - 256 || cols > FP8_MAX_COLS || (codes_t && rows > FP8_MAX_COLS)) return GROUTER_ERR_UNSUPPORTED;
  if (((int64_t)rows + 127) / 128 * (((int64_t)cols + 127) / 128) > INT32_MAX) return GROUTER_ERR_UNSUPPORTED;
  if ((!codes && !codes_t) || (codes && !scales) || (codes_t && !scales_t)) return rows && cols ? GROUTER_ERR_INVALID_ARG : GROUTER_OK;
  if (rows > 0 && cols > 0 && !x) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(x, dtype == GROUTER_F32 ? 4 : 2) || !aligned_to(codes, 16) || !aligned_to(scales, 16) || !aligned_to(codes_t, 16) ||
      !aligned_to(scales_t, 16))
    return GROUTER_ERR_MISALIGNED;
  if (rows == 0 || cols == 0) return GROUTER_OK;
  return launch_quantize(x, ldx, dtype, rows, cols, square != 0, codes, scales, codes_t, scales_t, nullptr, static_cast<cudaStream_t>(stream)) ==
                 cudaSuccess
             ? GROUTER_OK
             : GROUTER_ERR_CUDA;
}

int grouter_dequantize_fp8(const void* codes, const void* scales, int32_t rows, int32_t cols, int64_t ldy, int32_t dtype, void* y, void* stream) {
  if (rows < 0 || cols < 0 || ldy < cols || (dtype != GROUTER_BF16 && dtype != GROUTER_F32)) return GROUTER_ERR_INVALID_ARG;
  if (rows > INT32_MAX - 256 || cols > FP8_MAX_COLS) return GROUTER_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return GROUTER_OK;
  if (!codes || !scales || !y) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(codes, 16) || !aligned_to(scales, 16) || !aligned_to(y, dtype == GROUTER_F32 ? 4 : 2)) return GROUTER_ERR_MISALIGNED;
  const RowsGrid g = rows_grid(rows, cols);
  const bool vec = aligned_to(y, 16) && ldy % (dtype == GROUTER_F32 ? 4 : 8) == 0;
  const uint8_t *q = static_cast<const uint8_t*>(codes), *s = static_cast<const uint8_t*>(scales);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == GROUTER_F32
          ? launch_dependent(dequantize_kernel<float>, g.grid, dim3(Q_THREADS), 0, st, q, s, rows, cols, ldy, vec, g.shape, static_cast<float*>(y))
          : launch_dependent(dequantize_kernel<__nv_bfloat16>, g.grid, dim3(Q_THREADS), 0, st, q, s, rows, cols, ldy, vec, g.shape,
                             static_cast<__nv_bfloat16*>(y));
  return e == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
