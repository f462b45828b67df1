// Matrices into 8 bits and back (the format is in fp8.cuh): codes of the rows, of the transposed matrix, or both from one reading.
//
// Bound by HBM (2 bytes in and one out an element, two out with the transposed codes) as long as an element costs no more than the 17
// (rows) or 22 (both) instruction slots that its bytes leave it.  So bf16 stays in pairs: magnitudes are compared two to an instruction as
// 16-bit integers (their order is that of the numbers), infinities and NaN are looked for in the maximum only, and two elements are scaled
// and converted by one instruction each.
//   Rows alone: sixteen lanes (f32: 32) hold a block of 128, four rows in flight a thread.
//   Squares or transposed codes: a CTA takes a tile of 128 x 128, which is a block of every row, a block of every column and a whole
//     square.  For the transposed codes it waits in shared memory and is read by columns: a lane takes four neighbouring rows of a word's
//     columns (two of bf16), so that a column's codes leave as 128 bytes of a warp; words are permuted so that neither side meets
//     conflicts it need not have.
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

// Magnitudes in progress: of one f32 (as itself) or of two bf16 (as 16-bit halves of a word).
template <typename T>
__device__ __forceinline__ uint32_t word_top(uint32_t top, uint32_t w) {
  if constexpr (sizeof(T) == 4) return max(top, w & 0x7fffffffu);
  else return __vmaxu2(top, w & 0x7fff7fffu);
}
// ... without what is not finite
template <typename T>
__device__ __forceinline__ uint32_t word_top_finite(uint32_t top, uint32_t w) {
  if constexpr (sizeof(T) == 4) {
    w &= 0x7fffffffu;
    return w < 0x7f800000u ? max(top, w) : top;
  } else {
    w &= 0x7fff7fffu;
    if ((w & 0xffffu) >= 0x7f80u) w &= 0xffff0000u;
    if (w >= 0x7f800000u) w &= 0xffffu;
    return __vmaxu2(top, w);
  }
}
// the larger half of a pair, as the bits of an f32
template <typename T>
__device__ __forceinline__ uint32_t top_of_word(uint32_t top) {
  if constexpr (sizeof(T) == 4) return top;
  else return max(top << 16, top & 0xffff0000u);
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_top_bits(uint32_t v) {
  if constexpr (LANES == 32) return __reduce_max_sync(0xffffffffu, v);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ bool bits_not_finite(uint32_t top) { return top >= 0x7f800000u; }
// Elements 2j and 2j + 1 of some words, as f32.
template <typename T>
__device__ __forceinline__ float2 word_pair(const uint32_t* w, int j) {
  if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
  else return make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
}

// 16 bytes of row r from column c on; zeros outside the matrix.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load_row(const QuantParams& p, int64_t r, int c) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (r >= p.rows) return v;
  const T* at = static_cast<const T*>(p.x) + r * p.ldx + c;
  if constexpr (VEC) {
    if (c < p.cols) v = ld_stream16(at);
  } else {
    T* e = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int i = 0; i < vec16<T>(); ++i)
      if (c + i < p.cols) e[i] = at[i];
  }
  return v;
}

// Codes and the scale of the block that LANES neighbouring lanes hold 16 bytes each of; top: a magnitude known beforehand (a square's).
template <typename T, bool SQUARE>
__device__ __forceinline__ void put_row(const QuantParams& p, const uint4& v, int64_t r, int c, bool square_inf, uint32_t square, int64_t pitch, int64_t across) {
  constexpr int VE = vec16<T>(), LANES = QT / VE;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = square;
  bool inf = square_inf;
  if (!SQUARE) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = word_top<T>(top, w[i]);
    top = lanes_top_bits<LANES>(top_of_word<T>(top));
    inf = __any_sync(0xffffffffu, bits_not_finite(top));
    if (inf) {
      top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = word_top_finite<T>(top, w[i]);
      top = lanes_top_bits<LANES>(top_of_word<T>(top));
    }
  }
  const uint32_t e = fp8_exponent(__uint_as_float(top));
  const float2 inv = both(fp8_inverse(e));
  if (r < p.rows && c < pitch) {
    uint32_t q[VE / 4];
#pragma unroll
    for (int i = 0; i < VE / 4; ++i) {
      if (inf) q[i] = fp8_pair<true>(word_pair<T>(w, 2 * i), inv) | fp8_pair<true>(word_pair<T>(w, 2 * i + 1), inv) << 16;
      else q[i] = fp8_pair<false>(word_pair<T>(w, 2 * i), inv) | fp8_pair<false>(word_pair<T>(w, 2 * i + 1), inv) << 16;
    }
    uint8_t* to = p.codes + r * pitch + c;
    if constexpr (VE == 8) *reinterpret_cast<uint2*>(to) = make_uint2(q[0], q[1]);
    else *reinterpret_cast<uint32_t*>(to) = q[0];
    if ((c & (QT - 1)) == 0) p.scales[fp8_scale_at(r, c / QT, across)] = (uint8_t)e;
  }
}

// Codes of the rows alone.  A warp takes 512 bytes of four rows (bf16: two blocks a row), neighbouring warps neighbouring columns.
constexpr int QR_ROWS = 4;
template <typename T, bool VEC>
__global__ void __launch_bounds__(Q_THREADS) quantize_rows_kernel(const QuantParams p) {
  constexpr int VE = vec16<T>();
  const int64_t pitch = fp8_pitch(p.cols), across = fp8_atoms_across(p.cols);
  const int64_t chunks = (pitch + 32 * VE - 1) / (32 * VE);              // of a row
  const int64_t unit = (int64_t)blockIdx.x * (Q_THREADS / 32) + (threadIdx.x >> 5);
  const int64_t r0 = unit / chunks * QR_ROWS;
  const int c = (int)(unit % chunks) * (32 * VE) + (threadIdx.x & 31) * VE;
  after_previous_kernel();
  let_next_kernel_start();
  if (r0 >= p.rows) return;               // whole warps
  uint4 v[QR_ROWS];
#pragma unroll
  for (int n = 0; n < QR_ROWS; ++n) v[n] = load_row<T, VEC>(p, r0 + n, c);
#pragma unroll
  for (int n = 0; n < QR_ROWS; ++n) put_row<T, false>(p, v[n], r0 + n, c, false, 0u, pitch, across);
}

template <typename T, bool VEC, bool SQUARE>
__global__ void __launch_bounds__(Q_THREADS) quantize_tile_kernel(const QuantParams p) {
  constexpr int VE = vec16<T>(), LANES = QT / VE;                        // elements an access, lanes a row
  constexpr int STEP = Q_THREADS / LANES, NR = QT / STEP;                // rows a block at a time, times
  constexpr int WORDS = QT * (int)sizeof(T) / 4;                         // of a tile row
  extern __shared__ uint32_t s_tile[];    // [QT][WORDS], with transposed codes; word w of row r at w ^ (r / 4 % 32)
  __shared__ uint32_t s_top[2][Q_THREADS / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = threadIdx.x / LANES, at = threadIdx.x % LANES;
  const int64_t tr = blockIdx.x / p.tiles_c;
  const int tc = (int)(blockIdx.x - tr * p.tiles_c);
  const int64_t r0 = tr * QT;
  const int c0 = tc * QT, c = c0 + at * VE;
  after_previous_kernel();
  let_next_kernel_start();
  uint4 v[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) v[n] = load_row<T, VEC>(p, r0 + n * STEP + sub, c);
  uint32_t square = 0;
  bool square_inf = false;
  if (SQUARE) {
    auto block_top = [&](uint32_t t, int which) {
      t = lanes_top_bits<32>(top_of_word<T>(t));
      if (lane == 0) s_top[which][warp] = t;
      __syncthreads();
      t = s_top[which][0];
#pragma unroll
      for (int w = 1; w < Q_THREADS / 32; ++w) t = max(t, s_top[which][w]);
      return t;
    };
#pragma unroll
    for (int n = 0; n < NR; ++n) square = word_top<T>(word_top<T>(word_top<T>(word_top<T>(square, v[n].x), v[n].y), v[n].z), v[n].w);
    square = block_top(square, 0);
    square_inf = bits_not_finite(square);
    if (square_inf) {                     // the whole block alike
      square = 0;
#pragma unroll
      for (int n = 0; n < NR; ++n)
        square = word_top_finite<T>(word_top_finite<T>(word_top_finite<T>(word_top_finite<T>(square, v[n].x), v[n].y), v[n].z), v[n].w);
      square = block_top(square, 1);
    }
  }
  if (p.codes_t) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = n * STEP + sub, turn = r >> 2;
      uint32_t* row = s_tile + r * WORDS;
      row[(at * 4 + 0) ^ turn] = v[n].x;
      row[(at * 4 + 1) ^ turn] = v[n].y;
      row[(at * 4 + 2) ^ turn] = v[n].z;
      row[(at * 4 + 3) ^ turn] = v[n].w;
    }
  }
  if (p.codes) {
    const int64_t pitch = fp8_pitch(p.cols), across = fp8_atoms_across(p.cols);
#pragma unroll
    for (int n = 0; n < NR; ++n) put_row<T, SQUARE>(p, v[n], r0 + n * STEP + sub, c, square_inf, square, pitch, across);
  }
  if (p.codes_t) {
    __syncthreads();
    constexpr int CPW = 4 / (int)sizeof(T);
    const int64_t pitch = fp8_pitch(p.rows), across = fp8_atoms_across(p.rows);
    const bool here = r0 + 4 * lane < pitch;
#pragma unroll 4
    for (int wc = warp; wc < WORDS; wc += Q_THREADS / 32) {
      uint32_t q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = s_tile[(4 * lane + i) * WORDS + (wc ^ lane)];
      uint32_t word = 0;
      if (!SQUARE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) word = word_top<T>(word, q[i]);
      }
#pragma unroll
      for (int j = 0; j < CPW; ++j) {
        auto half = [&](uint32_t w) { return sizeof(T) == 4 ? w : j == 0 ? w << 16 : w & 0xffff0000u; };
        uint32_t top = square;
        bool inf = square_inf;
        if (!SQUARE) {
          top = lanes_top_bits<32>(half(word));
          inf = bits_not_finite(top);
          if (inf) {
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) some = word_top_finite<float>(some, half(q[i]));
            top = lanes_top_bits<32>(some);
          }
        }
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(half(q[i]));
        const uint32_t e = fp8_exponent(__uint_as_float(top));
        const float inv = fp8_inverse(e);
        const int col = c0 + wc * CPW + j;
        if (p.sums) {
          const float sum = lanes_sum<32>((f[0] + f[1]) + (f[2] + f[3]));
          if (lane == 0 && col < p.cols) p.sums[tr * p.cols + col] = sum;
        }
        if (col < p.cols && here) {
          *reinterpret_cast<uint32_t*>(p.codes_t + col * pitch + r0 + 4 * lane) = inf ? fp8_quad<true>(f, inv) : fp8_quad<false>(f, inv);
          if (lane == 0) p.scales_t[fp8_scale_at(col, (int)tr, across)] = (uint8_t)e;
        }
      }
    }
  }
}

// A thread's codes fill one 16-byte store (eight to bf16, four to f32), four rows' worth of them in flight; where the output's rows are not
// 16-byte aligned its elements are stored one by one.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int cols,
                                                         int64_t ldy, bool vec, T* __restrict__ y) {
  constexpr int VE = vec16<T>(), AHEAD = 4;
  const int64_t pitch = fp8_pitch(cols), per_row = pitch / VE, total = per_row * rows, across = fp8_atoms_across(cols);
  const int64_t step = (int64_t)gridDim.x * 256;
  after_previous_kernel();
  let_next_kernel_start();
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += AHEAD * step) {
    uint32_t w[AHEAD][VE / 4];
    float s[AHEAD];
    int64_t r[AHEAD];
    int c[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int64_t i = i0 + k * step;
      r[k] = i / per_row;
      c[k] = (int)(i - r[k] * per_row) * VE;
      if (i < total) {
        const uint8_t* from = codes + r[k] * pitch + c[k];
        if constexpr (VE == 8) *reinterpret_cast<uint2*>(w[k]) = __ldg(reinterpret_cast<const uint2*>(from));
        else w[k][0] = __ldg(reinterpret_cast<const uint32_t*>(from));
        s[k] = fp8_scale(__ldg(scales + fp8_scale_at(r[k], c[k] / FP8_BLOCK, across)));
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (i0 + k * step >= total) break;
      float f[VE];
#pragma unroll
      for (int i = 0; i < VE; i += 2) {
        const float2 t = mul2(fp8_values(w[k][i / 4] >> (8 * (i & 2))), both(s[k]));
        f[i] = t.x;
        f[i + 1] = t.y;
      }
      T* to = y + r[k] * ldy + c[k];
      if (vec && c[k] + VE <= cols) {
        st_pack<T, VE>(to, f);
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (c[k] + i < cols) to[i] = from_f32<T>(f[i]);
      }
    }
  }
}

namespace {

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
  const int64_t chunks = (fp8_pitch(p.cols) + 32 * vec16<T>() - 1) / (32 * vec16<T>()), warps = ((int64_t)p.rows + QR_ROWS - 1) / QR_ROWS * chunks;
  return launch_dependent(quantize_rows_kernel<T, VEC>, dim3((unsigned)((warps + Q_THREADS / 32 - 1) / (Q_THREADS / 32))), dim3(Q_THREADS), 0, st, p);
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
  if (rows > INT32_MAX - 256 || cols > INT32_MAX - 256) return GROUTER_ERR_UNSUPPORTED;
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
  if (rows > INT32_MAX - 256 || cols > INT32_MAX - 256) return GROUTER_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return GROUTER_OK;
  if (!codes || !scales || !y) return GROUTER_ERR_INVALID_ARG;
  if (!aligned_to(codes, 16) || !aligned_to(scales, 16) || !aligned_to(y, dtype == GROUTER_F32 ? 4 : 2)) return GROUTER_ERR_MISALIGNED;
  const int64_t work = fp8_pitch(cols) / (dtype == GROUTER_F32 ? 4 : 8) * rows, want = (work + 255) / 256, cap = (int64_t)current_sms() * 8;
  const dim3 grid((unsigned)(want < cap ? want : cap > 0 ? cap : 1));
  const bool vec = aligned_to(y, 16) && ldy % (dtype == GROUTER_F32 ? 4 : 8) == 0;
  const uint8_t *q = static_cast<const uint8_t*>(codes), *s = static_cast<const uint8_t*>(scales);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == GROUTER_F32
          ? launch_dependent(dequantize_kernel<float>, grid, dim3(256), 0, st, q, s, rows, cols, ldy, vec, static_cast<float*>(y))
          : launch_dependent(dequantize_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, q, s, rows, cols, ldy, vec, static_cast<__nv_bfloat16*>(y));
  return e == cudaSuccess ? GROUTER_OK : GROUTER_ERR_CUDA;
}

}  // extern "C"
