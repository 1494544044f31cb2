// The fifth-generation tensor cores of sm_100a in PTX: barriers, tensor copies, tensor memory, products.
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace dgc {

// Bound of a wait: a second, of which a time in which nothing of the GPU ran (another process's turn, a
// debugger) counts as a hundredth.
constexpr uint32_t kLongestWaitNs = 1000000000, kLongestStepNs = kLongestWaitNs / 100;

__device__ __forceinline__ uint32_t shared_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{.reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p;}" : "=r"(yes));
  return yes;
}

// ------------------------------------------------------------------ barriers
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_init_visible() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("{.reg .b64 s; mbarrier.arrive.shared::cta.b64 s, [%0];}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("{.reg .b64 s; mbarrier.arrive.expect_tx.shared::cta.b64 s, [%0], %1;}" ::"r"(bar), "r"(bytes) : "memory");
}
// The address of `local` in block `rank` of the cluster, and an arrival there.
__device__ __forceinline__ uint32_t in_block(uint32_t local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
  return r;
}
__device__ __forceinline__ void arrive_remote(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Whether the phase of this parity is over; the thread is suspended meanwhile, up to 20 us.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{.reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3; selp.u32 %0, 1, 0, p;}"
               : "=r"(done) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
  return done;
}
// Waits until the phase of this parity is over; false once it has taken too long, or another of the
// block's waits has (`failed`, in shared memory): the caller then leaves its loop.
static __device__ int g_waits_out;
struct Patience { uint64_t last; uint32_t spent; };
static __device__ __noinline__ bool too_long(Patience* p, volatile int* failed) {
  const uint64_t now = now_ns();
  if (p->last) p->spent += (uint32_t)min(now - p->last, (uint64_t)kLongestStepNs);
  p->last = now;
  if (*failed) return true;
  if (p->spent <= kLongestWaitNs) return false;
  *failed = 1;
  atomicAdd(&g_waits_out, 1);
  return true;
}
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* failed) {
  Patience p{0, 0};
  while (!try_wait(bar, parity))
    if (too_long(&p, failed)) return false;
  return true;
}
// The waits of this file's kernels that have run out since the last look, on the current device.
static inline int32_t take_waits_out(int* count) {
  DGC_CUDA(cudaMemcpyFromSymbol(count, g_waits_out, sizeof *count));
  const int none = 0;
  if (*count) DGC_CUDA(cudaMemcpyToSymbol(g_waits_out, &none, sizeof none));
  return DGC_OK;
}
// After a wait that ran out: time for the copies that are under way to end.
__device__ __forceinline__ void let_copies_end() {
  const uint64_t t = now_ns();
  for (int i = 0; i < 1 << 20 && now_ns() - t < kLongestStepNs; ++i) __nanosleep(1000);
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned; barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ------------------------------------------------------------------ pairs of 16-bit numbers, each operation rounded to the type
template <class T>
__device__ __forceinline__ uint32_t fma16(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
template <class T>
__device__ __forceinline__ uint32_t mul16(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <class T>
__device__ __forceinline__ uint32_t sub16(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>) asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <class T>
__device__ __forceinline__ uint32_t add16(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (std::is_same_v<T, __half>) asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// ------------------------------------------------------------------ tensor copies
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}
// GROUP 2: the barrier may be the other block's of the pair.
template <int GROUP>
__device__ __forceinline__ void load_tile(uint32_t to, const CUtensorMap* m, uint32_t bar, int x, int y, int z) {
  if constexpr (GROUP == 2)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(to), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(to), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void store_tile(const CUtensorMap* m, uint32_t from, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(from), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void shared_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ------------------------------------------------------------------ tensor memory
template <int GROUP>
__device__ __forceinline__ void tmem_alloc(uint32_t result, uint32_t columns) {
  if constexpr (GROUP == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}
template <int GROUP>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
  if constexpr (GROUP == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define DGC_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define DGC_I8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
// 32 columns of the warp's 32 lanes: a lane's thread gets its row.
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : DGC_R8(r, 0), DGC_R8(r, 8), DGC_R8(r, 16), DGC_R8(r, 24) : "r"(at));
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : DGC_R8(r, 0), DGC_R8(r, 8) : "r"(at));
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(at), DGC_I8(r, 0), DGC_I8(r, 8) : "memory");
}

// ------------------------------------------------------------------ products
// A tile in shared memory in the 128-byte swizzle, 1024-byte aligned.
//   rows of K: 8 rows of 128 bytes (64 elements of K) an atom, the next 8 rows 1024 bytes on; 16 elements
//     of K are 32 bytes.
//   rows of M or N: an atom is 8 elements of K, each a row of 64 elements; the next 8 of K 1024 bytes
//     on, the next 64 of M or N `groups` bytes on; 16 elements of K are 2048 bytes.
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t at, uint32_t groups) {
  return (uint64_t)((at & 0x3FFFF) >> 4) | (uint64_t)(groups >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// 16-bit operands, 32-bit sums; A or B `turned`: rows of M or N.
__host__ __device__ constexpr uint32_t product_descriptor(int m, int n, bool bf16, bool a_turned, bool b_turned) {
  return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (a_turned ? 1u : 0u) << 15 | (b_turned ? 1u : 0u) << 16 |
         (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
template <int GROUP>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  if constexpr (GROUP == 2)
    asm volatile("{.reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;}"
                 ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
  else
    asm volatile("{.reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;}"
                 ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
// The same with A in tensor memory (two 16-bit elements of a lane's row a column).
__device__ __forceinline__ void product_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{.reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;}"
               ::"r"(d), "r"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
// Arrives at the barrier (of both blocks of a pair) once this thread's products so far are done.
template <int GROUP>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (GROUP == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ------------------------------------------------------------------ host
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}
// A map of [z][y][x] 16-bit elements (strides in elements, multiples of 8; 16-byte aligned), tiles of 64 x box_y; what lies outside is read as 0 and not written.
inline int32_t tensor_map(CUtensorMap* m, const void* p, bool bf16, int64_t x, int64_t y, int64_t z, int64_t stride_y, int64_t stride_z,
                          int box_y) {
  const EncodeTiled f = encode_tiled();
  if (!f) return DGC_ECUDA;
  const cuuint64_t dims[3] = {(cuuint64_t)x, (cuuint64_t)y, (cuuint64_t)z};
  const cuuint64_t strides[2] = {(cuuint64_t)stride_y * 2, (cuuint64_t)stride_z * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_y, 1}, one[3] = {1, 1, 1};
  return f(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dims, strides, box, one,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? DGC_OK : DGC_ECUDA;
}

}  // namespace dgc
