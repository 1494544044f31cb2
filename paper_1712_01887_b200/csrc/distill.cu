// Distillation from a teacher's top logits (sm_100a): kernels and C ABI.
//
//   q = softmax over the row's listed teacher logits / T,  p = softmax(s / T),  p1 = softmax(s)
//   loss = w_soft T^2 sum_k q_k (log q_k - log p_{i_k})  +  w_hard (-log p1_y)
//   dloss / ds_j = w_soft T (p_j - sum_{k: i_k = j} q_k)  +  w_hard (p1_j - [j = y])
//
// A row is one block's work, or one cluster's where there are few rows.  One walk over the row
// keeps a running maximum and the sum(s) of exponentials under it per thread; the threads' pairs
// are joined by shuffles, shared memory and the cluster's shared memory.  The gradient's walk
// reads the row again (out of L2: the block has just read it) and writes p scaled; the few places
// that the list and the label name are then written once more with their q taken off.
//
// Exponentials are 2^(s c - round(m c)), c = log2(e) / T, m the row's maximum: the rounding of m c is
// the same factor in every term and cancels in p, and where the loss needs logarithms the same
// expression is used.  Below 2^24 that factor is within 2^-1/2 .. 2^1/2; rows whose m c or m log2(e)
// is larger (a mask of -1e9 or of the type's lowest value in every place: the factor of 1e10 can be
// 2^440, out of range) or that hold no finite number are done again as 2^((s - m) c).  Sums are
// 32-bit, two a thread (even and odd places), the rest is a tree: of a vocabulary of 262144 in one
// block a thread adds 512 terms to each, of 2^31 - 65 four million, whose roundings (at worst 2^-24
// of the sum each) are then no longer small.

#include <cooperative_groups.h>

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "rows.cuh"

namespace cg = cooperative_groups;
using namespace dgc;

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxCluster = 8;
constexpr float kDown = 0x1p-20f, kUp = 0x1p20f;        // logarithms on their way to the loss
constexpr float kLeast = 0x1p-110f, kMost = 0x1p110f;   // two sums kept from forward to backward
enum { kForward = 0, kBackward = 1, kBoth = 2 };

struct DistillArgs {
  const void* logits;
  void* dlogits;
  const int32_t* idx;
  const float* val;
  const int32_t* labels;
  const float* dloss;
  const float* stats_in;
  float *loss, *stats;
  int64_t ld, ld_d;
  float temperature, c, soft, hard;   // c = log2(e) / temperature
  float lowest;                       // maxima not above it, or not below its opposite, are taken with care
  int32_t vocab, k, cluster;
};

// A maximum and the sums of exponentials under it (s1: at temperature 1, where it differs).
// CAREFUL: exponents are (s - m) c, in any range; else s c - m c, see above.
template <bool TWO, bool CAREFUL>
struct Sums {
  float m, s = 0.0f, s1 = 0.0f;
  __device__ __forceinline__ explicit Sums(float lowest) : m(lowest) {}
  __device__ __forceinline__ void scale_to(float to, float c) {
    s *= exp2_fast(CAREFUL ? (m - to) * c : __fadd_rn(__fmul_rn(m, c), -__fmul_rn(to, c)));
    if (TWO) s1 *= exp2_fast(CAREFUL ? (m - to) * kLog2e : __fadd_rn(__fmul_rn(m, kLog2e), -__fmul_rn(to, kLog2e)));
    m = to;
  }
  // joins what the warp's lanes hold; every lane gets the result
  __device__ __forceinline__ void join(float c) {
    float top = m;
#pragma unroll
    for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    scale_to(top, c);
#pragma unroll
    for (int d = 16; d; d /= 2) {
      s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      if (TWO) s1 += __shfl_xor_sync(0xFFFFFFFFu, s1, d);
    }
  }
};

template <int NT>
struct DistillShared {
  float3 row[NT / 32], part[kMaxCluster];   // maximum, sum, sum at temperature 1
  float2 teacher[DGC_MAX_TOP / 32];
  float loss[DGC_MAX_TOP / 32];
  int idx[DGC_MAX_TOP];
  float q[DGC_MAX_TOP];
};

// Chunks of a thread under way at once, and blocks of 256 threads an SM.  The loss alone reads
// memory only: more blocks hide more (4096 x 50021 bf16: 72 us with five, 83 with four of more
// registers).  The gradient's second walk lives on L2, which more rows in work at once would not
// fit (168 us with four, 206 with five); 32-bit rows have half the arithmetic to a byte and gain
// from more loads instead (2048 x 32768: 104 us with eight and three, 120 with four and four).
template <class T, int MODE> constexpr int kAhead = sizeof(T) == 4 && MODE != kForward ? 8 : 4;
template <class T, int MODE> constexpr int kBlocks = MODE == kForward ? 5 : sizeof(T) == 4 ? 3 : 4;

template <class T, int NT, int MODE, bool TWO>
__global__ void __launch_bounds__(NT, kBlocks<T, MODE> * 256 / NT) k_distill(const DistillArgs a) {
  pdl_enter();
  constexpr int E = Row<T>::E, W = NT / 32, U = kAhead<T, MODE>;
  __shared__ DistillShared<NT> sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ncl = a.cluster;
  Part part = part_of(ncl);
  const int64_t r = part.row;
  const Row<T> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
  take_part(part, row, ncl);
  const int rank = part.rank, lo = part.lo, hi = part.hi;

  // the teacher's entry of thread k, the label: on their way while the row is walked
  int mine = -1, y = -1;
  float t = -INFINITY, sk = 0.0f, sy = 0.0f, w = 0.0f;
  if (tid < a.k) {
    mine = a.idx[r * a.k + tid];
    t = a.val[r * a.k + tid];
  }
  if (a.labels) y = a.labels[r];
  if (MODE != kForward) w = a.dloss[r];
  // and, after the walk, the student's logits there (the row is then in L2); without a soft term
  // (0 times an infinite loss would not be 0) nothing is listed
  const auto pick = [&] {
    if (mine < 0 || mine >= a.vocab || !(t > -INFINITY) || a.soft == 0.0f) mine = -1;
    else sk = to_float<T>(row.p[mine]);
    if (y < 0 || y >= a.vocab) y = -1;
    else sy = to_float<T>(row.p[y]);
  };

  // p = 2^(s c - mc) / sum,  p1 = 2^(s log2(e) - mc1) / sum1;  careful: 2^((s - m) c) and so on
  float m = 0.0f, mc = 0.0f, mc1 = 0.0f, sum = 1.0f, sum1 = 1.0f;
  bool careful = false, walk = MODE != kBackward;
  if (MODE == kBackward) {
    // What the forward call left: m c and the sum, so that p comes out as it would there; with two
    // sums, these as z 2^n each: p = 2^(s c - n) / z (a logarithm would cost p the bits before the
    // point).  Rows out of the ordinary have 0 there and are summed once more.
    const float x = a.stats_in[2 * r], x1 = a.stats_in[2 * r + 1];
    walk = TWO ? !(x > kLeast && x < kMost && x1 > kLeast && x1 < kMost) : !(x1 > 0.0f && x1 < kMost);
    mc = x;
    sum = x1;
    if (TWO) {
      const uint32_t u = __float_as_uint(x), u1 = __float_as_uint(x1);
      mc = (float)((int)(u >> 23) - 127);
      mc1 = (float)((int)(u1 >> 23) - 127);
      sum = __uint_as_float((u & 0x7FFFFFu) | 0x3F800000u);
      sum1 = __uint_as_float((u1 & 0x7FFFFFu) | 0x3F800000u);
    } else {
      sum1 = sum;
    }
  }
  // joins the threads' sums over the row's blocks
  const auto over_row = [&](auto st) {
    using S = decltype(st);
    st.join(a.c);
    if (lane == 0) sm.row[warp] = make_float3(st.m, st.s, st.s1);
    __syncthreads();
    const float lowest = sm.row[0].x;   // (any of the maxima will do for lanes without one)
    st = S(lowest);
    if (lane < W) { st.m = sm.row[lane].x; st.s = sm.row[lane].y; st.s1 = sm.row[lane].z; }
    st.join(a.c);
    if (ncl > 1) {
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();   // every block of the cluster runs
      if (tid < ncl) cl.map_shared_rank(&sm, tid)->part[rank] = make_float3(st.m, st.s, st.s1);
      cl.sync();
      st = S(sm.part[0].x);
      if (lane < ncl) { st.m = sm.part[lane].x; st.s = sm.part[lane].y; st.s1 = sm.part[lane].z; }
      st.join(a.c);
    }
    return st;
  };
  const auto teacher = [&] {   // (after the walk: the list's way from memory is then long over)
    if (warp * 32 < a.k) {
      Sums<false, true> te(-FLT_MAX);
      if (mine >= 0) { te.m = fmaxf(t, -FLT_MAX); te.s = 1.0f; }
      te.join(a.c);
      if (lane == 0) sm.teacher[warp] = make_float2(te.m, te.s);
    }
  };
  if (walk) {   // (the same for all threads of the row)
    Sums<TWO, false> st(a.lowest);
    Val<2> s2 = fill<2>(0.0f), s1 = fill<2>(0.0f);   // (sums of the even and the odd places)
    Val<2> minus = fill<2>(-__fmul_rn(st.m, a.c)), minus1 = fill<2>(-__fmul_rn(st.m, kLog2e));   // (rounded: see above)
    const Val<2> c = fill<2>(a.c), c1 = fill<2>(kLog2e);
    each_group<T, NT, U>(row, lo, hi, [&](const uint4 (&x)[U], int, int count) {
      uint32_t best = max_word<T, false>(x[0]);
#pragma unroll
      for (int u = 1; u < U; ++u)
        if (u < count) best = max_words<T, false>(best, max_word<T, false>(x[u]));
      const float top = max_of_word<T, false>(best);
      if (top > st.m) {
        const Val<2> now = fill<2>(-__fmul_rn(top, a.c)), now1 = fill<2>(-__fmul_rn(top, kLog2e));
        s2 = mul_(s2, fill<2>(exp2_fast(now.v[0] - minus.v[0])));
        if (TWO) s1 = mul_(s1, fill<2>(exp2_fast(now1.v[0] - minus1.v[0])));
        st.m = top;
        minus = now;
        minus1 = now1;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u >= max(count, 1)) continue;
        Val<2> v[E / 2];
        pairs_of<T>(x[u], v);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const Val<2> e = fma_(v[i], c, minus);
          s2 = add_(s2, Val<2>{{exp2_fast(e.v[0]), exp2_fast(e.v[1])}});
          if (TWO) {
            const Val<2> e1 = fma_(v[i], c1, minus1);
            s1 = add_(s1, Val<2>{{exp2_fast(e1.v[0]), exp2_fast(e1.v[1])}});
          }
        }
      }
    });
    pick();
    st.s = s2.v[0] + s2.v[1];
    st.s1 = s1.v[0] + s1.v[1];
    teacher();
    st = over_row(st);
    mc = st.m * a.c;
    mc1 = st.m * kLog2e;
    sum = st.s;
    sum1 = TWO ? st.s1 : st.s;
    careful = !(sum > 0.0f && fabsf(st.m) < -a.lowest);
    if (careful) {   // (the same for all threads of the row)
      __syncthreads();
      Sums<TWO, true> ca(-FLT_MAX);
      each_group<T, NT, 1>(row, lo, hi, [&](const uint4 (&x)[1], int, int) {
        Val<2> v[E / 2];
        pairs_of<T>(x[0], v);
        const float top = max_of_word<T, false>(max_word<T, false>(x[0]));
        if (top > ca.m) ca.scale_to(top, a.c);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float d = v[i / 2].v[i % 2] - ca.m;
          ca.s += exp2_fast(d * a.c);
          if (TWO) ca.s1 += exp2_fast(d * kLog2e);
        }
      });
      ca = over_row(ca);
      m = ca.m;
      sum = ca.s;
      sum1 = TWO ? ca.s1 : ca.s;
    }
  } else {
    pick();
    teacher();
    __syncthreads();
  }
  const auto exponent = [&](float v) { return careful ? (v - m) * a.c : fmaf(v, a.c, -mc); };
  const auto exponent1 = [&](float v) { return careful ? (v - m) * kLog2e : fmaf(v, kLog2e, -mc1); };
  // 2^-20 log p (a power of two changes no bit): a word masked with the type's lowest value has a finite log p,
  // whose exponent of two, or which itself before the weight, is out of range
  const auto log_of = [&](float v, float c, float minus, float total) {
    const float e = careful ? (kDown * v - kDown * m) * c : fmaf(kDown * v, c, -kDown * minus);
    return v == -INFINITY ? -INFINITY : e * kLn2 - kDown * logf(total);
  };

  float tm = -FLT_MAX, ts = 0.0f;   // the teacher's maximum and sum
  for (int i = 0; i * 32 < a.k; ++i) tm = fmaxf(tm, sm.teacher[i].x);
  for (int i = 0; i * 32 < a.k; ++i) ts += sm.teacher[i].y * exp2_fast((sm.teacher[i].x - tm) * a.c);
  const bool taught = !(ts <= 0.0f), labelled = y >= 0;   // (a teacher of +infinity: ts and q are NaN)
  float q = 0.0f;
  if (warp * 32 < a.k) {
    float logq = 0.0f;
    if (mine >= 0) {
      const float x = (fmaxf(t, -FLT_MAX) - tm) * a.c;
      q = __fdividef(exp2_fast(x), ts);
      logq = x * kLn2 - logf(ts);
    }
    if (MODE != kForward && tid < a.k) { sm.idx[tid] = mine; sm.q[tid] = q; }
    if (MODE != kBackward && rank == 0) {
      float kl = 0.0f;
      if (!(q <= 0.0f)) kl = q * (kDown * logq - log_of(sk, a.c, mc, sum));
#pragma unroll
      for (int d = 16; d; d /= 2) kl += __shfl_xor_sync(0xFFFFFFFFu, kl, d);
      if (lane == 0) sm.loss[warp] = kl;
    }
  }
  __syncthreads();   // (also: the listed logits are in registers, their places may be overwritten)
  if (MODE != kBackward && rank == 0 && tid == 0) {
    float soft = 0.0f;
    for (int i = 0; i * 32 < a.k; ++i) soft += sm.loss[i];
    float loss = taught ? a.soft * a.temperature * soft * a.temperature * kUp : 0.0f;
    if (labelled && a.hard != 0.0f)
      loss -= a.hard * log_of(sy, kLog2e, mc1, sum1) * kUp;
    a.loss[r] = loss;
    if (MODE == kForward && a.stats) {
      const auto total = [](float s, float e) {   // s 2^e, or 0: to be summed again
        const float n = rintf(e);
        return fabsf(e) < 100.0f ? ldexpf(s * exp2f(e - n), (int)n) : 0.0f;
      };
      a.stats[2 * r] = careful ? 0.0f : TWO ? total(sum, mc) : mc;
      a.stats[2 * r + 1] = careful ? 0.0f : TWO ? total(sum1, mc1) : sum;
    }
  }
  if (MODE == kForward) return;

  // gradient
  const float wq = taught ? w * a.soft * a.temperature : 0.0f;
  const float wy = labelled ? w * a.hard : 0.0f;
  float coef = __fdividef(wq, sum), coef1 = __fdividef(wy, sum1);
  if (sum == 0.0f) coef = coef1 = 0.0f;   // a row of -infinity: p is 0
  const bool zero = wq == 0.0f && wy == 0.0f;
  if (!TWO) coef += coef1;
  const auto grad = [&](float v) {
    float g = exp2_fast(exponent(v)) * coef;
    if (TWO) g = fmaf(exp2_fast(exponent1(v)), coef1, g);
    return g;
  };
  T* out = static_cast<T*>(a.dlogits) + r * a.ld_d;
  const bool same = (reinterpret_cast<uintptr_t>(out) & 15u) == (reinterpret_cast<uintptr_t>(row.p) & 15u);
  const auto put = [&](const Val<2> (&v)[E / 2], int e0, bool whole) {
    if (whole && same) {
      __stcs(reinterpret_cast<uint4*>(out + e0), chunk_of<T>(v));   // (not to be read again here: the rows are)
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (e0 + i >= 0 && e0 + i < a.vocab) store_one<T>(out + e0 + i, v[i / 2].v[i % 2]);
    }
  };
  if (careful || zero) {
    each_group<T, NT, 1>(row, lo, hi, [&](const uint4 (&x)[1], int j, int count) {
      Val<2> v[E / 2];
      pairs_of<T>(x[0], v);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i / 2].v[i % 2] = zero ? 0.0f : grad(v[i / 2].v[i % 2]);
      put(v, row.first(j), count > 0);
    });
  } else {
    const Val<2> c = fill<2>(a.c), minus = fill<2>(-mc), k = fill<2>(coef);
    const Val<2> c1 = fill<2>(kLog2e), minus1 = fill<2>(-mc1), k1 = fill<2>(coef1);
    each_group<T, NT, U>(row, lo, hi, [&](const uint4 (&x)[U], int j, int count) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u >= max(count, 1)) continue;
        Val<2> v[E / 2];
        pairs_of<T>(x[u], v);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const Val<2> e = fma_(v[i], c, minus);
          Val<2> g = mul_(Val<2>{{exp2_fast(e.v[0]), exp2_fast(e.v[1])}}, k);
          if (TWO) {
            const Val<2> e1 = fma_(v[i], c1, minus1);
            g = fma_(Val<2>{{exp2_fast(e1.v[0]), exp2_fast(e1.v[1])}}, k1, g);
          }
          v[i] = g;
        }
        put(v, row.first(j + u * NT), count > 0);
      }
    });
  }
  if (zero) return;
  __syncthreads();
  const int e_lo = max(row.first(lo), 0), e_hi = hi == row.chunks ? a.vocab : row.first(hi);
  if (mine >= e_lo && mine < e_hi) {
    bool first = true;
    float all = 0.0f;
    for (int j = 0; j < a.k; ++j) {
      if (sm.idx[j] == mine) {
        if (j < tid) first = false;
        all += sm.q[j];
      }
    }
    if (first) {
      const float g = grad(sk) - wq * all - (mine == y ? wy : 0.0f);
      store_one<T>(out + mine, g);
    }
  }
  if (tid == NT - 1 && y >= e_lo && y < e_hi) {
    bool listed = false;
    for (int j = 0; j < a.k; ++j) listed |= sm.idx[j] == y;
    if (!listed) store_one<T>(out + y, grad(sy) - wy);
  }
}

template <class T, int NT, int MODE, bool TWO>
int32_t go(const DistillArgs& a, int64_t rows, cudaStream_t s) {
  if (rows * a.cluster > INT32_MAX) return DGC_EINVAL;
  const dim3 grid((unsigned)(rows * a.cluster));
  if (a.cluster > 1) launch_cluster(k_distill<T, NT, MODE, TWO>, grid, NT, 0, s, (unsigned)a.cluster, a);
  else launch(k_distill<T, NT, MODE, TWO>, grid, NT, 0, s, a);
  return check_launch();
}

template <class T, int MODE, bool TWO>
int32_t choose(DistillArgs a, int64_t rows, cudaStream_t s) {
  // blocks for a row: few rows are spread over the SMs
  a.cluster = 1;
  while (a.cluster < kMaxCluster && rows * a.cluster < 148 && a.vocab / a.cluster > 8192) a.cluster *= 2;
  // a short row is little work beside what a warp does once a row
  if ((int64_t)a.vocab * (int)sizeof(T) <= 8192 && a.k <= 128) return go<T, 128, MODE, TWO>(a, rows, s);
  return go<T, 256, MODE, TWO>(a, rows, s);
}

template <class T>
int32_t enqueue(const DistillArgs& a, int mode, int64_t rows, cudaStream_t s) {
  const bool two = a.labels && a.hard != 0.0f && a.temperature != 1.0f;
  if (mode == kForward) return two ? choose<T, kForward, true>(a, rows, s) : choose<T, kForward, false>(a, rows, s);
  if (mode == kBackward) return two ? choose<T, kBackward, true>(a, rows, s) : choose<T, kBackward, false>(a, rows, s);
  return two ? choose<T, kBoth, true>(a, rows, s) : choose<T, kBoth, false>(a, rows, s);
}

int32_t distill(int mode, const dgc_distill* d, void* stream) {
  if (!d || bad_dtype(d->dtype) || d->rows < 0 || d->rows > INT32_MAX || d->vocab < 1 || d->vocab > INT32_MAX - 64 ||
      d->k < 1 || d->k > DGC_MAX_TOP)
    return DGC_EINVAL;
  // (T^2 and log2(e) / T are normal numbers then)
  if (!(d->temperature >= 0x1p-60f && d->temperature <= 0x1p60f) || !std::isfinite(d->soft_weight) ||
      !std::isfinite(d->hard_weight))
    return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  if (bad_matrix(d->logits, d->rows, d->vocab, es)) return DGC_EINVAL;
  if (mode != kForward && bad_matrix(d->dlogits, d->rows, d->vocab, es)) return DGC_EINVAL;
  if (d->rows == 0) return DGC_OK;
  if (!d->idx || !d->val || misaligned(d->idx, 4) || misaligned(d->val, 4) || misaligned(d->labels, 4) ||
      misaligned(d->loss, 4) || misaligned(d->stats, 4) || misaligned(d->dloss, 4))
    return DGC_EINVAL;
  if ((mode != kBackward && !d->loss) || (mode != kForward && !d->dloss) || (mode == kBackward && !d->stats)) return DGC_EINVAL;
  DistillArgs a{};
  a.logits = d->logits.data; a.ld = d->logits.ld; a.idx = d->idx; a.val = d->val; a.labels = d->labels;
  a.vocab = d->vocab; a.k = d->k; a.temperature = d->temperature; a.soft = d->soft_weight; a.hard = d->hard_weight;
  a.c = (float)(1.4426950408889634 / (double)d->temperature);
  a.lowest = -0x1p24f / std::max(kLog2e, a.c);
  a.loss = d->loss; a.stats = d->stats; a.stats_in = d->stats; a.dloss = d->dloss;
  a.dlogits = d->dlogits.data; a.ld_d = d->dlogits.ld;
  cudaStream_t s = as_stream(stream);
  if (d->dtype == DGC_F32) return enqueue<float>(a, mode, d->rows, s);
  if (d->dtype == DGC_BF16) return enqueue<__nv_bfloat16>(a, mode, d->rows, s);
  return enqueue<__half>(a, mode, d->rows, s);
}

}  // namespace

extern "C" {

int32_t dgc_distill_forward(const dgc_distill* d, void* stream) { return distill(kForward, d, stream); }
int32_t dgc_distill_backward(const dgc_distill* d, void* stream) { return distill(kBackward, d, stream); }
int32_t dgc_distill_loss_grad(const dgc_distill* d, void* stream) { return distill(kBoth, d, stream); }

}  // extern "C"
