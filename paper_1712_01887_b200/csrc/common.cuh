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

}  // namespace dgc
