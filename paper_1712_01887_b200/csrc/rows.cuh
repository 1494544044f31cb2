// Walking a row of a matrix in aligned 16-byte chunks, whatever address the row starts at
// (a vocabulary of odd size puts the rows of a 16-bit matrix at every 2-byte address).
#pragma once

#include "common.cuh"

namespace dgc {

// One row of n elements.  Chunk j is the j-th aligned 16-byte block that holds some of it:
// elements j * E - shift and the E - 1 after it.  Only the first and the last chunk can be
// partly outside the row; those are fetched element by element.
template <class T>
struct Row {
  static constexpr int E = 16 / sizeof(T);
  const T* p;
  const uint4* base;
  int n, shift, chunks;
  __device__ __forceinline__ Row(const T* row, int len) : p(row), n(len) {
    shift = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    base = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row) & ~(uintptr_t)15);
    chunks = (int)(((int64_t)len + shift + E - 1) / E);
  }
  __device__ __forceinline__ int first(int chunk) const { return chunk * E - shift; }
};

// A cluster's block: its row, its place, and its part [lo, hi) of the row's chunks.  (A division
// of 64-bit numbers here would cost a warp more than its share of a row of 10 KB.)
struct Part { int64_t row; int rank, lo, hi; };
__device__ __forceinline__ Part part_of(unsigned ncl) {
  if (ncl == 1) return Part{(int64_t)blockIdx.x, 0, 0, 0};
  return Part{(int64_t)(blockIdx.x / ncl), (int)(blockIdx.x % ncl), 0, 0};
}
template <class T>
__device__ __forceinline__ void take_part(Part& p, const Row<T>& row, unsigned ncl) {
  const int share = ncl == 1 ? row.chunks : (int)(((unsigned)row.chunks + ncl - 1) / ncl);
  p.lo = min(p.rank * share, row.chunks);
  p.hi = min(p.lo + share, row.chunks);
}

template <class T>
__device__ __forceinline__ void store_one(T* p, float v) {
  const float one[1] = {v};
  store_word<T, 1>(p, pack<T, 1>(one));
}

// -infinity in every place of a 32-bit word.
template <class T>
constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : std::is_same_v<T, __nv_bfloat16> ? 0xFF80FF80u : 0xFC00FC00u;

__device__ __forceinline__ void words_of(const uint4& w, uint32_t (&u)[4]) {
  u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
}

// Pairs of neighbouring elements of a chunk.
template <class T>
__device__ __forceinline__ void pairs_of(const uint4& w, Val<2> (&v)[8 / sizeof(T)]) {
  uint32_t u[4];
  words_of(w, u);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = Val<2>{{__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1])}};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack<T, 2>(u[i], v[i].v);
  }
}

template <class T>
__device__ __forceinline__ uint4 chunk_of(const Val<2> (&v)[8 / sizeof(T)]) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(v[0].v[0]), __float_as_uint(v[0].v[1]), __float_as_uint(v[1].v[0]),
                      __float_as_uint(v[1].v[1]));
  } else {
    return make_uint4(pack<T, 2>(v[0].v), pack<T, 2>(v[1].v), pack<T, 2>(v[2].v), pack<T, 2>(v[3].v));
  }
}

// The larger of two words, element by element.  NAN: a NaN wins, else it loses.
template <class T, bool NAN_WINS>
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (sizeof(T) == 4) {
    if (NAN_WINS) asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
    if (NAN_WINS) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  } else {
    if (NAN_WINS) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  }
  return r;
}
template <class T, bool NAN_WINS>
__device__ __forceinline__ uint32_t max_word(const uint4& w) {
  return max_words<T, NAN_WINS>(max_words<T, NAN_WINS>(w.x, w.y), max_words<T, NAN_WINS>(w.z, w.w));
}
template <class T, bool NAN_WINS>
__device__ __forceinline__ float max_of_word(uint32_t w) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(w);
  } else {
    float v[2];
    unpack<T, 2>(w, v);
    return __uint_as_float(max_words<float, NAN_WINS>(__float_as_uint(v[0]), __float_as_uint(v[1])));
  }
}

// The chunks among [lo, hi) that lie partly outside the row, for f as below.
template <class T, int NT, int U, class F>
__device__ __forceinline__ void odd_chunks(const Row<T>& r, int lo, int hi, bool tail, uint4 (&w)[U], F&& f) {
  constexpr int E = Row<T>::E;
  const int tid = threadIdx.x;
  int odd = -1;   // the chunks that are partly outside: one for thread 0, one for the last thread
  if (tid == 0 && lo == 0 && hi > 0 && r.shift) odd = 0;
  if (tid == NT - 1 && hi == r.chunks && lo < hi && tail && !(r.chunks == 1 && r.shift)) odd = r.chunks - 1;
  if (odd >= 0) {
    uint32_t u[4] = {kNone<T>, kNone<T>, kNone<T>, kNone<T>};
    const int e0 = r.first(odd);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = e0 + i;
      if (e >= 0 && e < r.n) {
        if constexpr (sizeof(T) == 4) {
          u[i] = *reinterpret_cast<const uint32_t*>(r.p + e);
        } else {
          const uint32_t h = *reinterpret_cast<const unsigned short*>(r.p + e);
          u[i / 2] = i % 2 ? (u[i / 2] & 0xFFFFu) | h << 16 : (u[i / 2] & 0xFFFF0000u) | h;
        }
      }
    }
    w[0] = make_uint4(u[0], u[1], u[2], u[3]);
    f(w, odd, 0);
  }
}

// f(chunks, first chunk, count) for the chunks [lo, hi) of a row, dealt to the block's NT threads
// in turn, U at a time: their loads are under way at once; chunk u is the first + u NT, and the
// first `count` are there.  A chunk that lies partly outside the row comes alone, as
// f(chunks, chunk, 0), with -infinity in the places outside.  Plain loads (not the read-only
// path): the gradient may be written over the logits.
// Groups for which `wanted()` is false are left out (it is asked once a group, in order; a chunk
// partly outside comes in any case).
template <class T, int NT, int U, class W, class F>
__device__ __forceinline__ void each_group_if(const Row<T>& r, int lo, int hi, W&& wanted, F&& f) {
  constexpr int E = Row<T>::E;
  const int tid = threadIdx.x;
  const bool tail = (r.n + r.shift) % E != 0;
  const int a = max(lo, r.shift ? 1 : 0), b = min(hi, r.chunks - (tail ? 1 : 0));
  uint4 w[U];
  int j = a + tid;
  for (; j + (U - 1) * NT < b; j += NT * U) {
    if (!wanted()) continue;
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = r.base[j + u * NT];
    f(w, j, U);
  }
  if (j < b && wanted()) {
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (j + u * NT < b) w[u] = r.base[j + u * NT];
    f(w, j, (b - 1 - j) / NT + 1);
  }
  odd_chunks<T, NT, U>(r, lo, hi, tail, w, f);
}

template <class T, int NT, int U, class F>
__device__ __forceinline__ void each_group(const Row<T>& r, int lo, int hi, F&& f) {
  each_group_if<T, NT, U>(r, lo, hi, [] { return true; }, f);
}

}  // namespace dgc
