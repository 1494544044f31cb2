// The k largest entries of every row of a matrix (sm_100a): kernel and C ABI.
//
// The list is in the library's form, (int32 index, fp32 value), largest value first and the
// lowest index first among equals.  A row is read once from memory:
//
//   1. every thread takes the maximum of the elements it is dealt, and of each group of them;
//   2. the k-th largest of the threads' maxima is a bound that at least k elements reach, and
//      that few others do (74 in all for k = 64 and 256 threads when the row is in no special
//      order), found bit by bit with a counting barrier each;
//   3. the groups whose maximum reaches it, and only those, are looked at again (out of L2),
//      and the elements that reach it are listed;
//   4. a listed entry's place is the number of listed entries that come before it.
//
// Where more entries reach the bound than the list holds (a row of equal values, an order that
// deals all large values to a few threads), the k-th value is found by bisection over the row,
// then its equals are taken in index order: slow, and always right.
//
// What bounds it: memory, and the latency of the steps between (4096 x 50021 bf16, k = 64: 91 us,
// 4.5 TB/s of the 6.6 measured for a copy).  Five blocks of 256 threads an SM hide that better than
// two of 512 (134 us); looking at whole rows again in step 3 took 107 us; the code that looks at one
// chunk is there once and not unrolled over a group (170 us: it did not fit the instruction cache).

#include <cooperative_groups.h>

#include <algorithm>

#include "rows.cuh"

namespace cg = cooperative_groups;
using namespace dgc;

namespace {

template <int NT> constexpr int kTopGroups = NT == 512 ? 4 : 8;
constexpr int kTopRank = 512;             // up to this many are ranked directly
constexpr uint32_t kLowest = 0x00800000u; // order key of the lowest finite value; -infinity is below

// Order key: larger float, larger key; -0 and +0 alike; NaN above everything.
__device__ __forceinline__ uint32_t order_key(float v) {
  v += 0.0f;
  const uint32_t b = __float_as_uint(v);
  if (v != v) return 0xFFFFFFFFu;
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0xFFFFFFFFu) return __uint_as_float(0x7FFFFFFFu);
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ unsigned long long entry(uint32_t key, int index) {
  return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)index);
}

template <int NT, int LIST>   // LIST: candidates a block can hold
struct TopShared {
  uint32_t groups[kTopGroups<NT>][NT];   // a thread's maxima by group of chunks; the last slot takes the rest
  unsigned long long list[LIST];
  unsigned long long best[DGC_MAX_TOP];
  uint2 range[32];
  int count, total[2];
};

// Sum over the block of a per-thread count.
template <int NT, int LIST>
__device__ __forceinline__ int block_sum(int v, TopShared<NT, LIST>& sm, int par) {
  v = __reduce_add_sync(0xFFFFFFFFu, v);
  if (threadIdx.x == 0) sm.total[par] = 0;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) atomicAdd(&sm.total[par], v);
  __syncthreads();
  return sm.total[par];
}

// A bound that at least k of the threads' keys reach if as many are above -infinity, and the
// lowest finite key otherwise: the k-th largest key, cut off below the bits that a type's
// rounding leaves (f32: ten bits of fraction are near enough).  The search starts below the bits
// that all keys have in common.
template <class T, int NT, int LIST>
__device__ __forceinline__ uint32_t kth_largest(uint32_t key, int k, TopShared<NT, LIST>& sm) {
  constexpr int low = std::is_same_v<T, __nv_bfloat16> ? 16 : 13;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool there = key >= kLowest;
  const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, key), bottom = __reduce_min_sync(0xFFFFFFFFu, there ? key : 0xFFFFFFFFu);
  if (lane == 0) sm.range[warp] = make_uint2(top, bottom);
  if (__syncthreads_count(there) < k) return kLowest;
  const uint2 mine = lane < NT / 32 ? sm.range[lane] : make_uint2(0, 0xFFFFFFFFu);
  const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, mine.x), lo = __reduce_min_sync(0xFFFFFFFFu, mine.y);
  int bit = 31 - __clz(hi ^ lo);                                   // -1: all alike
  uint32_t bound = bit < 0 ? lo : bit == 31 ? 0u : lo & ~((2u << bit) - 1u);
#pragma unroll 1
  for (; bit >= low; --bit) {
    const uint32_t c = bound | (1u << bit);
    if (__syncthreads_count(key >= c) >= k) bound = c;
  }
  return max(bound, kLowest);
}

// The k largest of the n listed entries (all different), in order, to sm.best.  Ends with a barrier.
template <int NT, int LIST>
__device__ void rank_list(TopShared<NT, LIST>& sm, int n, int k) {
  const int tid = threadIdx.x;
  unsigned long long floor = 0;   // entries below it are out
  if (n > kTopRank && n > k) {
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long c = floor | (1ull << bit);
      int mine = 0;
      for (int i = tid; i < n; i += NT) mine += sm.list[i] >= c;
      if (block_sum<NT>(mine, sm, bit & 1) >= k) floor = c;
    }
  }
  for (int i = tid; i < n; i += NT) {
    const unsigned long long e = sm.list[i];
    if (e < floor) continue;
    int before = 0;
    for (int j = 0; j < n; ++j) before += sm.list[j] > e;
    if (before < k) sm.best[before] = e;
  }
  __syncthreads();
}

// The row's part [lo, hi) in chunks: its k largest entries above -infinity, in order, to
// sm.best; returns how many there are.
template <class T, int NT, int LIST>
__device__ int top_of_part(const Row<T>& row, int lo, int hi, int k, TopShared<NT, LIST>& sm) {
  constexpr int E = Row<T>::E, U = NT == 512 ? 8 : 6;
  const int tid = threadIdx.x;
  uint32_t best = kNone<T>;   // (two maxima of 16-bit types; a NaN wins)
  int group = 0;
  each_group<T, NT, U>(row, lo, hi, [&](const uint4 (&w)[U], int, int count) {
    uint32_t here = max_word<T, true>(w[0]);
#pragma unroll
    for (int u = 1; u < U; ++u)
      if (u < count) here = max_words<T, true>(here, max_word<T, true>(w[u]));
    if (count > 0) {
      if (group < kTopGroups<NT>) sm.groups[group][tid] = here;
      else sm.groups[kTopGroups<NT> - 1][tid] = max_words<T, true>(here, sm.groups[kTopGroups<NT> - 1][tid]);
      ++group;
    }
    best = max_words<T, true>(best, here);
  });
  const uint32_t key = order_key(max_of_word<T, true>(best));
  const uint32_t bound = kth_largest<T, NT>(key, k, sm);
  if (tid == 0) sm.count = 0;
  __syncthreads();
  const auto list_above = [&](uint32_t from) {
    const float floor = key_value(from);
    const auto list = [&](const uint4& w, int e0) {
      Val<2> v[E / 2];
      pairs_of<T>(w, v);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float x = v[i / 2].v[i % 2];
        if (!(x < floor) && order_key(x) >= from) {   // (a NaN floor or x is not less)
          const int at = atomicAdd(&sm.count, 1);
          if (at < LIST) sm.list[at] = entry(order_key(x), e0 + i);
        }
      }
    };
    const auto reaches = [&](uint32_t w) { return !(max_of_word<T, true>(w) < floor); };
    int g = 0;
    each_group_if<T, NT, U>(row, lo, hi, [&] { return reaches(sm.groups[min(g++, kTopGroups<NT> - 1)][tid]); },
                            [&](const uint4 (&w)[U], int j, int count) {
      if (count == 0) {
        list(w[0], row.first(j));
        return;
      }
      uint32_t which = 0;   // chunks to look at one by one: few, so the code for one is there once
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u < count && reaches(max_word<T, true>(w[u]))) which |= 1u << u;
      for (; which; which &= which - 1) {
        const int chunk = j + (__ffs(which) - 1) * NT;
        list(row.base[chunk], row.first(chunk));
      }
    });
  };
  if (key >= bound) list_above(bound);
  __syncthreads();
  int n = sm.count;
  __syncthreads();
  if (n > LIST) {
    // bisection for the k-th value: `good` is reached by k entries or more, `bad` by fewer
    uint32_t good = bound, bad = 0xFFFFFFFFu;
    int par = 0;
    auto reach = [&](uint32_t from) {
      int mine = 0;
      each_group<T, NT, 2>(row, lo, hi, [&](const uint4 (&w)[2], int, int count) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (u >= max(count, 1)) continue;
          Val<2> v[E / 2];
          pairs_of<T>(w[u], v);
#pragma unroll
          for (int i = 0; i < E; ++i) mine += order_key(v[i / 2].v[i % 2]) >= from;
        }
      });
      return block_sum<NT>(mine, sm, par ^= 1);
    };
    if (reach(bad) >= k) good = bad;   // k NaN
    while (bad - good > 1) {
      const uint32_t mid = good + (bad - good) / 2;
      if (reach(mid) >= k) good = mid;
      else bad = mid;
    }
    if (tid == 0) sm.count = 0;
    __syncthreads();
    if (good != 0xFFFFFFFFu) list_above(good + 1);   // fewer than k
    __syncthreads();
    n = sm.count;
    // the k-th value's equals in index order, until the list is full
    for (int j0 = lo; j0 < hi && n < k; j0 += NT) {
      const int j = j0 + tid;
      uint32_t hit = 0;
      const int e0 = row.first(min(j, hi));
      if (j < hi) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const int e = e0 + i;
          if (e >= 0 && e < row.n && order_key(to_float<T>(row.p[e])) == good) hit |= 1u << i;
        }
      }
      // places in order: hits of the warps before, then of the lanes before
      const int lane = tid & 31, warp = tid >> 5;
      int before = __popc(hit);
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, before, d);
        if (lane >= d) before += o;
      }
      __shared__ int warps[NT / 32];
      if (lane == 31) warps[warp] = before;
      __syncthreads();
      int base = n, all = 0;
      for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) base += warps[w];
        all += warps[w];
      }
      base += before - __popc(hit);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (hit >> i & 1) {
          if (base < k) sm.list[base] = entry(good, e0 + i);
          ++base;
        }
      }
      n = min(k, n + all);
      __syncthreads();
    }
  }
  rank_list<NT>(sm, n, k);
  return min(n, k);
}

// One cluster a row: its blocks take parts of the row, the first block joins their lists.
template <class T, int NT, int LIST>
__global__ void __launch_bounds__(NT, NT == 128 ? 8 : NT == 256 ? 5 : 2)
k_top_logits(const T* logits, int64_t ld, int32_t rows, int32_t vocab, int32_t k, int32_t ncl,
             int32_t* idx, float* val) {
  pdl_enter();
  __shared__ TopShared<NT, LIST> sm;
  Part part = part_of(ncl);
  const int64_t r = part.row;
  const Row<T> row(logits + r * ld, vocab);
  take_part(part, row, ncl);
  const int rank = part.rank, lo = part.lo, hi = part.hi;
  int n = top_of_part<T, NT>(row, lo, hi, k, sm);
  if (ncl > 1) {
    // every block writes the entries of its own part that are among the row's k largest: their
    // places are the numbers of larger entries in all parts' lists, which are in order
    cg::cluster_group cl = cg::this_cluster();
    if (threadIdx.x == 0) sm.total[0] = n;
    cl.sync();
    for (int i = threadIdx.x; i < ncl * k; i += NT) {
      TopShared<NT, LIST>* peer = cl.map_shared_rank(&sm, i / k);
      sm.list[i] = i % k < peer->total[0] ? peer->best[i % k] : 0;   // (0: below every entry)
    }
    cl.sync();   // the peers' lists have been read
    int all = 0;
    for (int i = threadIdx.x; i < n; i += NT) {
      const unsigned long long e = sm.best[i];
      int place = i;
      for (int q = 0; q < ncl; ++q) {
        if (q == rank) continue;
        const unsigned long long* list = sm.list + q * k;
        int a = 0, b = k;      // list[0, a) > e, list[b, k) < e
        while (a < b) {
          const int m = (a + b) / 2;
          if (list[m] > e) a = m + 1;
          else b = m;
        }
        place += a;
      }
      if (place < k) {
        idx[r * k + place] = (int32_t)(0xFFFFFFFFu - (uint32_t)e);
        val[r * k + place] = key_value((uint32_t)(e >> 32));
      }
    }
    if (rank != 0) return;
    for (int q = threadIdx.x; q < ncl * k; q += NT) all += sm.list[q] != 0;
    all = block_sum<NT>(all, sm, 1);
    for (int i = all + threadIdx.x; i < k; i += NT) {   // fewer than k in the whole row
      idx[r * k + i] = -1;
      val[r * k + i] = -INFINITY;
    }
    return;
  }
  for (int i = threadIdx.x; i < k; i += NT) {
    const unsigned long long e = i < n ? sm.best[i] : 0;
    idx[r * k + i] = i < n ? (int32_t)(0xFFFFFFFFu - (uint32_t)e) : -1;
    val[r * k + i] = i < n ? key_value((uint32_t)(e >> 32)) : -INFINITY;
  }
}

template <class T, int NT, int LIST>
int32_t go(const dgc_top& d, int ncl, cudaStream_t s) {
  const int64_t grid = d.rows * ncl;
  if (grid > INT32_MAX) return DGC_EINVAL;
  if (ncl > 1)
    launch_cluster(k_top_logits<T, NT, LIST>, dim3((unsigned)grid), NT, 0, s, (unsigned)ncl, static_cast<const T*>(d.logits.data),
                   d.logits.ld, (int32_t)d.rows, d.vocab, d.k, ncl, d.idx, d.val);
  else
    launch(k_top_logits<T, NT, LIST>, dim3((unsigned)grid), NT, 0, s, static_cast<const T*>(d.logits.data), d.logits.ld,
           (int32_t)d.rows, d.vocab, d.k, ncl, d.idx, d.val);
  return check_launch();
}

template <class T>
int32_t enqueue(const dgc_top& d, cudaStream_t s) {
  // few rows are spread over the SMs: 8 blocks for each of 3 rows of 250007 (f32) take 13 us, one 57
  int ncl = 1;
  while (ncl < 8 && d.rows * ncl < 148 && d.vocab / ncl > 16384) ncl *= 2;
  // Threads: few for short rows (8000 x 1000 bf16: 77 us with 128, 92 with 256), many for long lists, whose
  // bound is the tighter the more maxima there are, and where a row's time counts.
  if ((int64_t)d.vocab * (int)sizeof(T) <= 8192 && d.k <= 128) return go<T, 128, 1024>(d, ncl, s);
  if (ncl > 1 || d.k > 128) return go<T, 512, 4096>(d, ncl, s);
  return go<T, 256, 2048>(d, ncl, s);
}

}  // namespace

extern "C" int32_t dgc_top_logits(const dgc_top* d, void* stream) {
  if (!d || bad_dtype(d->dtype) || d->rows < 0 || d->rows > INT32_MAX || d->vocab < 1 || d->vocab > INT32_MAX - 64 ||
      d->k < 1 || d->k > DGC_MAX_TOP || bad_matrix(d->logits, d->rows, d->vocab, element_size(d->dtype)))
    return DGC_EINVAL;
  if (d->rows == 0) return DGC_OK;
  if (!d->idx || !d->val || misaligned(d->idx, 4) || misaligned(d->val, 4)) return DGC_EINVAL;
  if (d->dtype == DGC_F32) return enqueue<float>(*d, as_stream(stream));
  if (d->dtype == DGC_BF16) return enqueue<__nv_bfloat16>(*d, as_stream(stream));
  return enqueue<__half>(*d, as_stream(stream));
}
