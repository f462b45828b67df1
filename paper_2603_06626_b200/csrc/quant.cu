// Matrices into 8 bits and back (the format is in fp8.cuh): codes of the rows, of the transposed matrix, or both from one reading.
//
// A block takes a tile of 128 x 128 elements, which is a block of every row, a block of every column, and a whole square.  Rows are
// quantized as they arrive, sixteen lanes (f32: 32) to a row; for the transposed codes the tile waits in shared memory and is read
// by columns.  Bound by HBM: 2 bytes in and one out an element, two out with the transposed codes.
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

// Words of a tile row in shared memory: one more than the row takes, so that neighbouring rows start in neighbouring banks.
template <typename T>
__host__ __device__ constexpr int q_pitch() { return QT * (int)sizeof(T) / 4 + 1; }

template <typename T, bool VEC, bool SQUARE>
__global__ void __launch_bounds__(Q_THREADS) quantize_kernel(const QuantParams p) {
  constexpr int VE = vec16<T>(), LANES = QT / VE;      // elements an access, lanes a row
  constexpr int STEP = Q_THREADS / LANES, NR = QT / STEP;                // rows a block at a time, times
  extern __shared__ uint32_t s_tile[];    // [QT][q_pitch], with transposed codes
  __shared__ uint32_t s_top[Q_THREADS / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = threadIdx.x / LANES, at = threadIdx.x % LANES;
  const int64_t tr = blockIdx.x / p.tiles_c;
  const int tc = (int)(blockIdx.x - tr * p.tiles_c);
  const int64_t r0 = tr * QT;
  const int c0 = tc * QT, c = c0 + at * VE;
  const T* x = static_cast<const T*>(p.x);
  after_previous_kernel();
  let_next_kernel_start();
  Pack<T, VE> v[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int64_t r = r0 + n * STEP + sub;
#pragma unroll
    for (int i = 0; i < VE; ++i) v[n].v[i] = from_f32<T>(0.f);
    if (r < p.rows) {
      if (VEC) {
        if (c < p.cols) v[n] = ld_pack<T, VE>(x + r * p.ldx + c);
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (c + i < p.cols) v[n].v[i] = x[r * p.ldx + c + i];
      }
    }
  }
  uint32_t square = 0;
  if (SQUARE) {
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int i = 0; i < VE; ++i) square = max(square, finite_magnitude(to_f32(v[n].v[i])));
    square = lanes_max_bits<32>(square);
    if (lane == 0) s_top[warp] = square;
    __syncthreads();
    square = s_top[0];
#pragma unroll
    for (int w = 1; w < Q_THREADS / 32; ++w) square = max(square, s_top[w]);
  }
  if (p.codes) {
    const int64_t pitch = fp8_pitch(p.cols), across = fp8_atoms_across(p.cols);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int64_t r = r0 + n * STEP + sub;
      float f[VE];
      uint32_t top = square;
#pragma unroll
      for (int i = 0; i < VE; ++i) f[i] = to_f32(v[n].v[i]);
      if (!SQUARE) {
#pragma unroll
        for (int i = 0; i < VE; ++i) top = max(top, finite_magnitude(f[i]));
        top = lanes_max_bits<LANES>(top);
      }
      const uint32_t e = fp8_exponent(top);
      const float inv = fp8_inverse(e);
      if (r < p.rows && c < pitch) {
        uint8_t* to = p.codes + r * pitch + c;
        if constexpr (VE == 8) *reinterpret_cast<uint2*>(to) = make_uint2(fp8_quad(f, inv), fp8_quad(f + 4, inv));
        else *reinterpret_cast<uint32_t*>(to) = fp8_quad(f, inv);
        if (at == 0) p.scales[fp8_scale_at(r, tc, across)] = (uint8_t)e;
      }
    }
  }
  if (p.codes_t) {
    constexpr int P = q_pitch<T>(), W = VE * (int)sizeof(T) / 4;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&v[n]);
#pragma unroll
      for (int i = 0; i < W; ++i) s_tile[(n * STEP + sub) * P + at * W + i] = w[i];
    }
    __syncthreads();
    // a lane takes four neighbouring rows of a word's columns (two of bf16, one of f32): a column's codes leave as 128 bytes of a warp
    constexpr int CPW = 4 / (int)sizeof(T);
    const int64_t pitch = fp8_pitch(p.rows), across = fp8_atoms_across(p.rows);
    for (int wc = warp; wc < QT / CPW; wc += Q_THREADS / 32) {
      uint32_t q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = s_tile[(4 * lane + i) * P + wc];
#pragma unroll
      for (int j = 0; j < CPW; ++j) {
        float f[4];
        uint32_t top = square;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[i] = __uint_as_float(sizeof(T) == 4 ? q[i] : j == 0 ? q[i] << 16 : q[i] & 0xffff0000u);
          if (!SQUARE) top = max(top, finite_magnitude(f[i]));
        }
        if (!SQUARE) top = lanes_max_bits<32>(top);
        const uint32_t e = fp8_exponent(top);
        const int col = c0 + wc * CPW + j;
        if (p.sums) {
          const float sum = lanes_sum<32>((f[0] + f[1]) + (f[2] + f[3]));
          if (lane == 0 && col < p.cols) p.sums[tr * p.cols + col] = sum;
        }
        if (col < p.cols && r0 + 4 * lane < pitch) {
          *reinterpret_cast<uint32_t*>(p.codes_t + col * pitch + r0 + 4 * lane) = fp8_quad(f, fp8_inverse(e));
          if (lane == 0) p.scales_t[fp8_scale_at(col, (int)tr, across)] = (uint8_t)e;
        }
      }
    }
  }
}

// Sixteen codes a thread; where the output's rows are not 16-byte aligned its elements are stored one by one.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int cols,
                                                         int64_t ldy, bool vec, T* __restrict__ y) {
  after_previous_kernel();
  let_next_kernel_start();
  const int64_t pitch = fp8_pitch(cols), per_row = pitch / 16, total = per_row * rows, across = fp8_atoms_across(cols);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row;
    const int c = (int)(i - r * per_row) * 16;
    const uint4 q = ld_stream16(codes + r * pitch + c);
    const float s = fp8_scale(__ldg(scales + fp8_scale_at(r, c / FP8_BLOCK, across)));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    float f[16];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 t = fp8_values(w[k / 2] >> (16 * (k & 1)));
      f[2 * k] = t.x * s;
      f[2 * k + 1] = t.y * s;
    }
    T* to = y + r * ldy + c;
    if (vec && c + 16 <= cols) {
#pragma unroll
      for (int k = 0; k < 16; k += vec16<T>()) st_pack<T, vec16<T>()>(to + k, f + k);
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (c + k < cols) to[k] = from_f32<T>(f[k]);
    }
  }
}

namespace {

template <typename T, bool VEC, bool SQUARE>
cudaError_t quantize_launch(const QuantParams& p, cudaStream_t st) {
  constexpr int smem = QT * q_pitch<T>() * 4;
  auto kern = quantize_kernel<T, VEC, SQUARE>;
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
  if (dtype == GROUTER_F32) {
    if (vec) return square ? quantize_launch<float, true, true>(p, st) : quantize_launch<float, true, false>(p, st);
    return square ? quantize_launch<float, false, true>(p, st) : quantize_launch<float, false, false>(p, st);
  }
  if (vec) return square ? quantize_launch<__nv_bfloat16, true, true>(p, st) : quantize_launch<__nv_bfloat16, true, false>(p, st);
  return square ? quantize_launch<__nv_bfloat16, false, true>(p, st) : quantize_launch<__nv_bfloat16, false, false>(p, st);
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
  const int64_t work = fp8_pitch(cols) / 16 * rows, want = (work + 255) / 256, cap = (int64_t)current_sms() * 8;
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
