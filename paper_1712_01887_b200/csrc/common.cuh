// What every translation unit of the library shares: the launch helpers (host), the stream
// order of programmatic launches and the conversion of the element types (device).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <type_traits>

#include "dgc.h"

#define DGC_CUDA(call)                         \
  do {                                         \
    cudaError_t e__ = (call);                  \
    if (e__ != cudaSuccess) {                  \
      (void)cudaGetLastError();                \
      return e__ == cudaErrorMemoryAllocation ? DGC_ENOMEM : DGC_ECUDA; \
    }                                          \
  } while (0)

namespace dgc {

inline std::atomic<uint64_t> g_launches{0};

inline cudaStream_t as_stream(void* s) { return reinterpret_cast<cudaStream_t>(s); }

// Launch with the programmatic-dependent-launch attribute (see pdl_enter).
template <class... KArgs, class... Args>
inline void launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s,
                   Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);   // error: check_launch()
}

// The same with a thread-block cluster of `cluster` blocks along x.
template <class... KArgs, class... Args>
inline void launch_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                           cudaStream_t s, unsigned cluster, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);   // error: check_launch()
}

// Lets a kernel have `bytes` of dynamic shared memory; the driver is asked once per kernel and
// device.
template <auto KERNEL>
inline int32_t allow_shared(size_t bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  DGC_CUDA(cudaGetDevice(&dev));
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return DGC_OK;
  DGC_CUDA(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  done.fetch_or(bit, std::memory_order_relaxed);
  return DGC_OK;
}

// Whether the device runs the kernel in clusters of more than the portable eight blocks; asked
// once per kernel and device.
template <auto KERNEL>
inline bool allow_cluster(int blocks, int threads, size_t shared) {
  static std::atomic<uint64_t> asked{0}, yes{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= 64) return (void)cudaGetLastError(), false;
  const uint64_t bit = 1ull << dev;
  if (!(asked.load(std::memory_order_acquire) & bit)) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = blocks;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = shared;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
        cudaOccupancyMaxActiveClusters(&n, KERNEL, &cfg) == cudaSuccess && n > 0)
      yes.fetch_or(bit, std::memory_order_relaxed);
    (void)cudaGetLastError();
    asked.fetch_or(bit, std::memory_order_release);
  }
  return yes.load(std::memory_order_relaxed) & bit;
}

// Whether a matrix argument of rows x cols cannot be what it says.
inline bool bad_matrix(const dgc_matrix& m, int64_t rows, int64_t cols, size_t elem) {
  return m.ld < cols || (rows > 0 && (!m.data || (reinterpret_cast<uintptr_t>(m.data) & (elem - 1)) != 0));
}
inline bool misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }
inline size_t element_size(int32_t dtype) { return dtype == DGC_F32 ? 4 : 2; }
inline bool bad_dtype(int32_t dtype) { return dtype < DGC_F32 || dtype > DGC_F16; }

inline int32_t check_launch() {
  g_launches.fetch_add(1, std::memory_order_relaxed);
  cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? DGC_OK : DGC_ECUDA;
}

// Stream order of the library's kernels: each is launched with the programmatic-serialization
// attribute and starts with this wait, which returns once the preceding kernel in the stream
// has completed and its writes are visible.
__device__ __forceinline__ void pdl_enter() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ------------------------------------------------------------------ element types
// Words of VEC elements (4 bytes, or one 2-byte element where a row is not 4-byte aligned).
template <class T, int VEC>
__device__ __forceinline__ uint32_t load_word(const T* p) {
  static_assert(sizeof(T) * VEC == 4 || sizeof(T) * VEC == 2, "");
  if constexpr (sizeof(T) * VEC == 4) return __ldg(reinterpret_cast<const uint32_t*>(p));
  else return __ldg(reinterpret_cast<const unsigned short*>(p));
}

template <class T, int VEC>
__device__ __forceinline__ void store_word(T* p, uint32_t w) {
  if constexpr (sizeof(T) * VEC == 4) *reinterpret_cast<uint32_t*>(p) = w;
  else *reinterpret_cast<unsigned short*>(p) = (unsigned short)w;
}

template <class T, int VEC>
__device__ __forceinline__ void unpack(uint32_t w, float (&v)[VEC]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(w);
  } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
    v[0] = __uint_as_float(w << 16);
    if constexpr (VEC == 2) v[1] = __uint_as_float(w & 0xFFFF0000u);
  } else {
    v[0] = __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu)));
    if constexpr (VEC == 2) v[1] = __half2float(__ushort_as_half((unsigned short)(w >> 16)));
  }
}

template <class T>
__device__ __forceinline__ uint32_t round_one(float v) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(v);
  else if constexpr (std::is_same_v<T, __nv_bfloat16>) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
  else return __half_as_ushort(__float2half_rn(v));
}

// Rounds once, to nearest even: the results leave 32 bits only here.
template <class T, int VEC>
__device__ __forceinline__ uint32_t pack(const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    return round_one<T>(v[0]);
  } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&p);
  } else {
    const __half2 p = __floats2half2_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
}

template <class T>
__device__ __forceinline__ T from_float(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else if constexpr (std::is_same_v<T, __nv_bfloat16>) return __float2bfloat16_rn(v);
  else return __float2half_rn(v);
}

template <class T>
__device__ __forceinline__ float to_float(T v) {
  if constexpr (sizeof(T) == 4) return v;
  else if constexpr (std::is_same_v<T, __nv_bfloat16>) return __bfloat162float(v);
  else return __half2float(v);
}

// ------------------------------------------------------------------ packed arithmetic
// One or two numbers, with the packed 32-bit arithmetic of sm_100 (two operations an instruction,
// each rounded as its scalar form).
template <int VEC> struct alignas(4 * VEC) Val { float v[VEC]; };

__device__ __forceinline__ unsigned long long bits(const Val<2>& a) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.v[0]), "f"(a.v[1]));
  return r;
}
__device__ __forceinline__ Val<2> val(unsigned long long r) {
  Val<2> a;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a.v[0]), "=f"(a.v[1]) : "l"(r));
  return a;
}
template <int VEC>
__device__ __forceinline__ Val<VEC> fill(float x) {
  Val<VEC> r;
#pragma unroll
  for (int i = 0; i < VEC; ++i) r.v[i] = x;
  return r;
}
__device__ __forceinline__ Val<2> fma_(const Val<2>& a, const Val<2>& b, const Val<2>& c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return val(r);
}
__device__ __forceinline__ Val<2> mul_(const Val<2>& a, const Val<2>& b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return val(r);
}
__device__ __forceinline__ Val<2> add_(const Val<2>& a, const Val<2>& b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return val(r);
}
__device__ __forceinline__ Val<1> fma_(const Val<1>& a, const Val<1>& b, const Val<1>& c) { return {{fmaf(a.v[0], b.v[0], c.v[0])}}; }
__device__ __forceinline__ Val<1> mul_(const Val<1>& a, const Val<1>& b) { return {{a.v[0] * b.v[0]}}; }
__device__ __forceinline__ Val<1> add_(const Val<1>& a, const Val<1>& b) { return {{a.v[0] + b.v[0]}}; }
// a - b
template <int VEC>
__device__ __forceinline__ Val<VEC> sub_(const Val<VEC>& a, const Val<VEC>& b) { return fma_(b, fill<VEC>(-1.0f), a); }

// 2^x, to 2 ulp; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace dgc
