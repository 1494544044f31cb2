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

template <class T>
__device__ __forceinline__ void store_one(T* p, float v) {
  const float one[1] = {v};
  store_word<T, 1>(p, pack<T, 1>(one));
}

template <class T>
__device__ __forceinline__ void unpack_chunk(const uint4& w, float (&v)[16 / sizeof(T)]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      v[i] = __uint_as_float(u[i]);
    } else {
      float pair[2];
      unpack<T, 2>(u[i], pair);
      v[2 * i] = pair[0];
      v[2 * i + 1] = pair[1];
    }
  }
}

template <class T>
__device__ __forceinline__ uint4 pack_chunk(const float (&v)[16 / sizeof(T)]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      u[i] = __float_as_uint(v[i]);
    } else {
      const float pair[2] = {v[2 * i], v[2 * i + 1]};
      u[i] = pack<T, 2>(pair);
    }
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// f(values, first element, whole) for the chunks [lo, hi) of a row, dealt to the block's NT
// threads in turn; U loads of a thread are under way at once.  Places outside the row hold
// -infinity, and `whole` is false for their chunks.  Plain loads (not the read-only path): the
// gradient may be written over the logits.
template <class T, int NT, int U, class F>
__device__ __forceinline__ void each_chunk(const Row<T>& r, int lo, int hi, F&& f) {
  constexpr int E = Row<T>::E;
  const int tid = threadIdx.x;
  const bool tail = (r.n + r.shift) % E != 0;
  const int a = max(lo, r.shift ? 1 : 0), b = min(hi, r.chunks - (tail ? 1 : 0));
  for (int j = a + tid; j < b; j += NT * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j + u * NT < b) w[u] = r.base[j + u * NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j + u * NT < b) {
        float v[E];
        unpack_chunk<T>(w[u], v);
        f(v, r.first(j + u * NT), true);
      }
    }
  }
  int odd = -1;   // the chunks that are partly outside: one for thread 0, one for the last thread
  if (tid == 0 && lo == 0 && hi > 0 && r.shift) odd = 0;
  if (tid == NT - 1 && hi == r.chunks && lo < hi && tail && !(r.chunks == 1 && r.shift)) odd = r.chunks - 1;
  if (odd >= 0) {
    float v[E];
    const int e0 = r.first(odd);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = e0 + i;
      v[i] = e >= 0 && e < r.n ? to_float<T>(r.p[e]) : -INFINITY;
    }
    f(v, e0, false);
  }
}

}  // namespace dgc
