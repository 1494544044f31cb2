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
// Exponentials are 2^((s - m) c), c = log2(e) / T, with m the row's maximum: the difference comes
// first, so that rows of very large or very low logits (a mask of the type's lowest value in
// every place) lose nothing and cannot overflow.  Sums are 32-bit: a thread adds at most a few
// hundred terms, the rest is a tree.

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
constexpr float kLseExact = 64.0f;   // 32-bit logarithms up to here give p to 4e-6
enum { kForward = 0, kBackward = 1, kBoth = 2 };

struct DistillArgs {
  const void* logits;
  void* dlogits;
  const int32_t* idx;
  const float* val;
  const int32_t* labels;
  const float* dloss;
  const float* lse_in;
  float *loss, *lse;
  int64_t ld, ld_d;
  float temperature, c, soft, hard;   // c = log2(e) / temperature
  int32_t vocab, k, cluster;
};

// Running maximum and sums of exponentials under it (s1: at temperature 1, where it differs).
// The maximum starts at the lowest finite value, so that rows of -infinity sum to zero.
template <bool TWO>
struct Sums {
  float m = -FLT_MAX, s = 0.0f, s1 = 0.0f;
  __device__ __forceinline__ void scale_to(float to, float c) {
    s *= exp2_fast((m - to) * c);
    if (TWO) s1 *= exp2_fast((m - to) * kLog2e);
    m = to;
  }
  // joins the pairs of `width` neighbouring lanes; every lane gets the result
  __device__ __forceinline__ void join(int width, float c) {
    float top = m;
    for (int d = width / 2; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    scale_to(top, c);
    for (int d = width / 2; d; d /= 2) {
      s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      if (TWO) s1 += __shfl_xor_sync(0xFFFFFFFFu, s1, d);
    }
  }
};

template <int NT>
struct DistillShared {
  float3 row[NT / 32], part[kMaxCluster];   // maximum, sum, sum at temperature 1
  float2 teacher[NT / 32];
  float loss[NT / 32];
  int idx[DGC_MAX_TOP];
  float q[DGC_MAX_TOP];
};

template <class T, int NT, int MODE, bool TWO>
#ifndef DB
#define DB 2
#endif
__global__ void __launch_bounds__(NT, DB * 512 / NT) k_distill(const DistillArgs a) {
  pdl_enter();
  constexpr int E = Row<T>::E, W = NT / 32, U = 4;
  __shared__ DistillShared<NT> sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ncl = a.cluster, rank = ncl > 1 ? (int)(blockIdx.x % ncl) : 0;
  const int64_t r = blockIdx.x / ncl;
  const Row<T> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
  const int lo = (int)((int64_t)row.chunks * rank / ncl), hi = (int)((int64_t)row.chunks * (rank + 1) / ncl);

  // the teacher's entry and the student's logit of thread k, the label
  int mine = -1;
  float t = -INFINITY, sk = 0.0f, sy = 0.0f;
  if (tid < a.k) {
    mine = a.idx[r * a.k + tid];
    t = a.val[r * a.k + tid];
    if (mine < 0 || mine >= a.vocab || !(t > -INFINITY)) mine = -1;
    else sk = to_float<T>(row.p[mine]);
  }
  int y = a.labels ? a.labels[r] : -1;
  if (y < 0 || y >= a.vocab) y = -1;
  else sy = to_float<T>(row.p[y]);
  const float w = MODE == kForward ? 0.0f : a.dloss[r];

  Sums<false> te;
  if (mine >= 0) { te.m = fmaxf(t, -FLT_MAX); te.s = 1.0f; }
  te.join(32, a.c);
  if (lane == 0) sm.teacher[warp] = make_float2(te.m, te.s);

  // p = 2^((s - m) c) / sum,  p1 = 2^((s - m1) log2 e) / sum1
  float m = 0.0f, m1 = 0.0f, sum = 1.0f, sum1 = 1.0f;
  bool walk = MODE != kBackward;
  if (MODE == kBackward) {
    const float2 lse = make_float2(a.lse_in[2 * r], a.lse_in[2 * r + 1]);
    m = lse.x * a.temperature;
    m1 = lse.y;
    // 32 bits of a large logarithm are too few for p: such rows are summed once more
    walk = !(fabsf(lse.x) < kLseExact && fabsf(lse.y) < kLseExact);
  }
  if (walk) {   // (the same for all threads of the row)
    Sums<TWO> st;
    Val<2> s2 = fill<2>(0.0f), s1 = fill<2>(0.0f);   // (sums of the even and the odd places)
    each_group<T, NT, U>(row, lo, hi, [&](const uint4 (&x)[U], int, int count) {
      uint32_t best = max_word<T, false>(x[0]);
#pragma unroll
      for (int u = 1; u < U; ++u)
        if (u < count) best = max_words<T, false>(best, max_word<T, false>(x[u]));
      const float top = max_of_word<T, false>(best);
      if (top > st.m) {
        s2 = mul_(s2, fill<2>(exp2_fast((st.m - top) * a.c)));
        if (TWO) s1 = mul_(s1, fill<2>(exp2_fast((st.m - top) * kLog2e)));
        st.m = top;
      }
      const Val<2> minus = fill<2>(-st.m);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u >= max(count, 1)) continue;
        Val<2> v[E / 2];
        pairs_of<T>(x[u], v);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const Val<2> d = add_(v[i], minus), e = mul_(d, fill<2>(a.c));
          s2 = add_(s2, Val<2>{{exp2_fast(e.v[0]), exp2_fast(e.v[1])}});
          if (TWO) {
            const Val<2> e1 = mul_(d, fill<2>(kLog2e));
            s1 = add_(s1, Val<2>{{exp2_fast(e1.v[0]), exp2_fast(e1.v[1])}});
          }
        }
      }
    });
    st.s = s2.v[0] + s2.v[1];
    st.s1 = s1.v[0] + s1.v[1];
    st.join(32, a.c);
    if (lane == 0) sm.row[warp] = make_float3(st.m, st.s, st.s1);
    __syncthreads();
    st = Sums<TWO>();
    if (lane < W) { st.m = sm.row[lane].x; st.s = sm.row[lane].y; st.s1 = sm.row[lane].z; }
    st.join(32, a.c);
    if (ncl > 1) {
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();   // every block of the cluster runs
      if (tid < ncl) cl.map_shared_rank(&sm, tid)->part[rank] = make_float3(st.m, st.s, st.s1);
      cl.sync();
      st = Sums<TWO>();
      if (lane < ncl) { st.m = sm.part[lane].x; st.s = sm.part[lane].y; st.s1 = sm.part[lane].z; }
      st.join(32, a.c);
    }
    m = m1 = st.m;
    sum = st.s;
    sum1 = TWO ? st.s1 : st.s;
  } else {
    __syncthreads();
  }
  te = Sums<false>();
  if (lane < W) { te.m = sm.teacher[lane].x; te.s = sm.teacher[lane].y; }
  te.join(32, a.c);

  const bool taught = te.s > 0.0f, labelled = y >= 0;
  float q = 0.0f, logq = 0.0f;
  if (mine >= 0) {
    const float x = (fmaxf(t, -FLT_MAX) - te.m) * a.c;
    q = __fdividef(exp2_fast(x), te.s);
    logq = x * kLn2 - logf(te.s);
  }
  if (MODE != kBackward && rank == 0) {
    float part = 0.0f;
    if (!(q <= 0.0f)) {
      const float logp = sk == -INFINITY ? -INFINITY : (sk - m) * a.c * kLn2 - logf(sum);
      part = q * (logq - logp);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) part += __shfl_xor_sync(0xFFFFFFFFu, part, d);
    if (lane == 0) sm.loss[warp] = part;
    __syncthreads();
    if (tid == 0) {
      float soft = 0.0f;
      for (int i = 0; i < W; ++i) soft += sm.loss[i];
      float loss = taught ? a.soft * a.temperature * a.temperature * soft : 0.0f;
      if (labelled && a.hard != 0.0f)
        loss -= a.hard * (sy == -INFINITY ? -INFINITY : (sy - m1) - logf(sum1));
      a.loss[r] = loss;
      if (MODE == kForward && a.lse) {
        a.lse[2 * r] = sum == 0.0f ? -INFINITY : m / a.temperature + logf(sum);
        a.lse[2 * r + 1] = TWO ? (sum1 == 0.0f ? -INFINITY : m1 + logf(sum1)) : a.lse[2 * r];
      }
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
  auto grad = [&](float v) {
    float g = exp2_fast((v - m) * a.c) * coef;
    if (TWO) g = fmaf(exp2_fast((v - m1) * kLog2e), coef1, g);
    return g;
  };
  if (tid < a.k) { sm.idx[tid] = mine; sm.q[tid] = q; }
  T* out = static_cast<T*>(a.dlogits) + r * a.ld_d;
  const bool same = (reinterpret_cast<uintptr_t>(out) & 15u) == (reinterpret_cast<uintptr_t>(row.p) & 15u);
  __syncthreads();   // the listed logits are in registers: their places may be overwritten
  each_group<T, NT, U>(row, lo, hi, [&](const uint4 (&x)[U], int j, int count) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u >= max(count, 1)) continue;
      Val<2> v[E / 2];
      pairs_of<T>(x[u], v);
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const Val<2> s = v[i], e = mul_(add_(s, fill<2>(-m)), fill<2>(a.c));
        v[i] = mul_(Val<2>{{exp2_fast(e.v[0]), exp2_fast(e.v[1])}}, fill<2>(coef));
        if (TWO) {
          const Val<2> e1 = mul_(add_(s, fill<2>(-m1)), fill<2>(kLog2e));
          v[i] = fma_(Val<2>{{exp2_fast(e1.v[0]), exp2_fast(e1.v[1])}}, fill<2>(coef1), v[i]);
        }
        if (zero) v[i] = fill<2>(0.0f);
      }
      const int e0 = row.first(j + u * NT);
      if (count > 0 && same) {
        *reinterpret_cast<uint4*>(out + e0) = chunk_of<T>(v);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (e0 + i >= 0 && e0 + i < a.vocab) store_one<T>(out + e0 + i, v[i / 2].v[i % 2]);
      }
    }
  });
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

template <class T, int MODE, bool TWO>
void go(const DistillArgs& a, int64_t rows, cudaStream_t s) {
  const dim3 grid((unsigned)(rows * a.cluster));
  if (a.vocab <= 4096) launch_cluster(k_distill<T, 256, MODE, TWO>, grid, 256, 0, s, (unsigned)a.cluster, a);
#ifndef DNT
#define DNT 512
#endif
  else launch_cluster(k_distill<T, DNT, MODE, TWO>, grid, DNT, 0, s, (unsigned)a.cluster, a);
}

template <class T>
int32_t enqueue(DistillArgs a, int mode, int64_t rows, cudaStream_t s) {
  a.cluster = 1;
  while (a.cluster < kMaxCluster && rows * a.cluster < 148 && a.vocab / a.cluster > 8192) a.cluster *= 2;
  if (rows * a.cluster > INT32_MAX) return DGC_EINVAL;
  const bool two = a.labels && a.hard != 0.0f && a.temperature != 1.0f;
  if (mode == kForward) two ? go<T, kForward, true>(a, rows, s) : go<T, kForward, false>(a, rows, s);
  else if (mode == kBackward) two ? go<T, kBackward, true>(a, rows, s) : go<T, kBackward, false>(a, rows, s);
  else two ? go<T, kBoth, true>(a, rows, s) : go<T, kBoth, false>(a, rows, s);
  return check_launch();
}

int32_t distill(int mode, const dgc_distill* d, void* stream) {
  if (!d || bad_dtype(d->dtype) || d->rows < 0 || d->rows > INT32_MAX || d->vocab < 1 || d->vocab > INT32_MAX - 64 ||
      d->k < 1 || d->k > DGC_MAX_TOP)
    return DGC_EINVAL;
  if (!(d->temperature > 0.0f) || !std::isfinite(d->temperature) || !std::isfinite(d->soft_weight) ||
      !std::isfinite(d->hard_weight))
    return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  if (bad_matrix(d->logits, d->rows, d->vocab, es)) return DGC_EINVAL;
  if (mode != kForward && bad_matrix(d->dlogits, d->rows, d->vocab, es)) return DGC_EINVAL;
  if (d->rows == 0) return DGC_OK;
  if (!d->idx || !d->val || misaligned(d->idx, 4) || misaligned(d->val, 4) || misaligned(d->labels, 4) ||
      misaligned(d->loss, 4) || misaligned(d->lse, 4) || misaligned(d->dloss, 4))
    return DGC_EINVAL;
  if ((mode != kBackward && !d->loss) || (mode != kForward && !d->dloss) || (mode == kBackward && !d->lse)) return DGC_EINVAL;
  DistillArgs a{};
  a.logits = d->logits.data; a.ld = d->logits.ld; a.idx = d->idx; a.val = d->val; a.labels = d->labels;
  a.vocab = d->vocab; a.k = d->k; a.temperature = d->temperature; a.soft = d->soft_weight; a.hard = d->hard_weight;
  a.c = (float)(1.4426950408889634 / (double)d->temperature);
  a.loss = d->loss; a.lse = d->lse; a.lse_in = d->lse; a.dloss = d->dloss;
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
