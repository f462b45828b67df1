// Typed loads and stores of a few consecutive elements, shared by the kernels around the expert layer (layer norm,
// balance loss, optimizer): bf16 or f32 in memory, f32 in registers, 16 bytes at a time where VE elements fill them.
#pragma once
#include "common.cuh"

namespace grouter {

// Streaming multiprocessors of the current device (0 without one); looked up once a device.
inline int current_sms() {
  static int sms[64] = {};
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev >= 0 && dev < 64 && sms[dev]) return sms[dev];
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev >= 0 && dev < 64) sms[dev] = n;
  return n;
}

// Launches a kernel that may be scheduled while the kernel before it on the stream still runs (programmatic dependent launch).  It calls
// after_previous_kernel() before it touches anything, or, launched with waits_at_end, before it ends.
//
// waits_at_end: such a kernel works beside the end of a run of kernels.  For the runs that the operators launch this holds, and has to hold
// when one of them is changed:
//   - A run begins with a kernel that waits at its start, before it lets the next one start.  All that came before it on the stream is then
//     complete for every kernel of the run, however early it is scheduled: each of them starts after all blocks of the one before have
//     let it, and so, going back, after the first one's wait.
//   - No kernel of the run reads or overwrites what another one of it writes, nor writes what another one reads.
//   - Each kernel after the first waits for the one before it at its end, so that the last one's end is the end of all: whatever waits for
//     that one at its start (a sum of pieces, the next call) may read what any of them wrote.
template <typename... Params, typename... Args>
inline cudaError_t launch_dependent(void (*kern)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<Params>(args)...);
}
// Waits until the kernel before this one on the stream has ended (and so, as each waits for the one before it, all before that) and its
// writes are visible.
__device__ __forceinline__ void after_previous_kernel() { cudaGridDependencySynchronize(); }
// From here on, once every block of this kernel has come here or ended, the next kernel's blocks may be scheduled.  What they may touch before
// this kernel's end is said at launch_dependent.
__device__ __forceinline__ void let_next_kernel_start() { cudaTriggerProgrammaticLaunchCompletion(); }

inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Elements of T in one 16-byte access.
template <typename T>
__host__ __device__ constexpr int vec16() { return 16 / (int)sizeof(T); }

// VE elements as they lie in memory, fetched in one access where that is a power-of-two size up to 16 bytes.
template <typename T, int VE>
struct alignas(VE * sizeof(T) <= 16 ? VE * sizeof(T) : 16) Pack {
  T v[VE];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Streamed once: read-only path, no L1 line kept.
__device__ __forceinline__ uint4 ld_stream16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Asynchronous copies of 16 or 8 bytes from global to shared memory, in groups of the issuing thread.
__device__ __forceinline__ void copy16_async(void* smem, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(global) : "memory");
}
__device__ __forceinline__ void copy8_async(void* smem, const void* global) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T, int VE>
__device__ __forceinline__ Pack<T, VE> ld_pack(const T* p) {
  Pack<T, VE> r;
  if constexpr (VE * sizeof(T) == 16) {
    *reinterpret_cast<uint4*>(&r) = ld_stream16(p);
  } else if constexpr (VE * sizeof(T) == 8) {
    *reinterpret_cast<uint2*>(&r) = __ldg(reinterpret_cast<const uint2*>(p));
  } else if constexpr (VE == 2) {
    *reinterpret_cast<uint32_t*>(&r) = __ldg(reinterpret_cast<const uint32_t*>(p));
  } else {
    static_assert(VE == 1, "whole 16-byte accesses, pairs or single elements");
    r.v[0] = __ldg(p);
  }
  return r;
}
// Elements 2j and 2j + 1 of an array of packs, as f32.  Two bf16 come out of their word in one instruction each.
template <typename T, int VE, int N>
__device__ __forceinline__ float2 pair_at(const Pack<T, VE> (&q)[N], int j) {
  if constexpr (VE == 1) {
    return make_float2(to_f32(q[2 * j].v[0]), to_f32(q[2 * j + 1].v[0]));
  } else if constexpr (sizeof(T) == 2) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&q[2 * j / VE])[(2 * j % VE) / 2];
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  } else {
    return make_float2(q[2 * j / VE].v[2 * j % VE], q[2 * j / VE].v[2 * j % VE + 1]);
  }
}
// VE values rounded to T, two bf16 to an instruction.
template <typename T, int VE>
__device__ __forceinline__ Pack<T, VE> make_pack(const float* f) {
  Pack<T, VE> r;
  if constexpr (VE > 1 && sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < VE; i += 2) reinterpret_cast<__nv_bfloat162*>(&r)[i / 2] = __floats2bfloat162_rn(f[i], f[i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i) r.v[i] = from_f32<T>(f[i]);
  }
  return r;
}
template <typename T, int VE>
__device__ __forceinline__ void st_pack(T* p, const float* f) {
  *reinterpret_cast<Pack<T, VE>*>(p) = make_pack<T, VE>(f);
}

// Two f32 operations in one instruction (each rounded by itself).
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmul.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n.reg .b64 x, y, z, w;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\nfma.rn.f32x2 w, x, y, z;\nmov.b64 {%0, %1}, w;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Column sums of n_part rows of `cols` values in a fixed order; the first n0 columns go to out0, the others to out1 (or nowhere).
cudaError_t launch_sum_rows(const float* partial, int n_part, int cols, float* out0, int n0, float* out1, cudaStream_t st);

}  // namespace grouter
