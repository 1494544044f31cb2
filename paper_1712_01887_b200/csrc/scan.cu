// Gated linear recurrence over packed sequences (sm_100a): kernels and C ABI.
//
//   f_t = 1 / (1 + exp(-z_t)),   h_t = f_t h_{t-1} + (1 - f_t) x_t        per channel
//
// Both directions of the computation are first-order linear recurrences, and such a recurrence
// over a run of steps is the map  y_out = P y_in + S  (P the product of the coefficients, S the
// result from y_in = 0), so runs can be reduced side by side and joined afterwards:
//
//   forward    y = h,           P = prod f,  S: h = f h + (1 - f) x
//   backward   e_t = f_t g_t,   g_t = dh_t + e_{t+1}:  the same map, walked from the end
//
// A lane owns one 32-bit word of a row (two 16-bit channels, or one of 32 bits) and a warp L
// consecutive steps of 32 such words, kept in registers.  A block of NW warps holds NW*L steps;
// a cluster of blocks holds consecutive ones.  Every thread reduces its run to (P, S), the runs
// are joined in order through shared memory (the blocks' through the cluster's), and the second
// walk over the registers starts from the true state.  The words of the next steps are loaded
// before the join, so memory stays busy while the blocks talk.  One pass over the data, no
// workspace, and a fixed order of the additions: results do not vary from run to run.
//
// A sequence is one cluster's work, so nothing (no infinity, no NaN) can cross from one
// sequence into its neighbour in the pack.

#include <cooperative_groups.h>

#include <algorithm>

#include "common.cuh"

namespace cg = cooperative_groups;
using namespace dgc;

namespace {

constexpr int kMaxCluster = 8;

struct ScanArgs {
  const void *z, *x, *dh, *h_in;
  void *h, *dz, *dx;
  const float *h0, *dh_last;
  float *h_last, *dh0;
  const int32_t* seq_start;
  int64_t ld_z, ld_x, ld_h, ld_dh, ld_dz, ld_dx;
  int32_t tokens, seqs, seq_len, channels, ctiles, cluster, reverse;
};

// sigma(z) and 1 - sigma(z), each to full relative precision (1 - f is not formed by
// subtraction: for gates near 1 it is the weight of the input).
__device__ __forceinline__ void gate(float z, float& f, float& omf) {
  const float e = __expf(-fabsf(z));
  const float big = __fdividef(1.0f, 1.0f + e);
  const float small = e * big;
  f = z >= 0.0f ? big : small;
  omf = z >= 0.0f ? small : big;
}

__device__ __forceinline__ void sequence_range(const ScanArgs& a, int s, int& first, int& len) {
  if (a.seq_start) {   // offsets are clamped: a damaged table cannot lead outside the tensors
    int lo = __ldg(a.seq_start + s), hi = __ldg(a.seq_start + s + 1);
    lo = min(max(lo, 0), a.tokens);
    hi = min(max(hi, lo), a.tokens);
    first = lo;
    len = hi - lo;
  } else {
    first = s * a.seq_len;
    len = a.seq_len;
  }
}

// Joins the runs of all warps of the cluster in order.  `carry` is the state before the first
// run on entry and after the last on return; the return value `mine` is the state before this
// warp's run.  `par` alternates from call to call: a buffer is written again only after
// everyone has passed the barrier of the call in between, hence has read it.
template <int VEC, int NW>
struct Join {
  float2 runs[2][NW][32][VEC];
  float2 blocks[2][kMaxCluster][32][VEC];
};

template <int VEC, int NW>
__device__ __forceinline__ void join_runs(Join<VEC, NW>& sm, int par, int ncl, int rank, int warp,
                                          int lane, const float (&P)[VEC], const float (&S)[VEC],
                                          float (&carry)[VEC], float (&mine)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) sm.runs[par][warp][lane][v] = make_float2(P[v], S[v]);
  __syncthreads();
  if (ncl > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (warp < ncl) {   // warp w hands this block's map to block w of the cluster
      float2 t[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) t[v] = make_float2(1.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float2 r = sm.runs[par][w][lane][v];
          t[v] = make_float2(r.x * t[v].x, fmaf(r.x, t[v].y, r.y));
        }
      }
      Join<VEC, NW>* peer = cl.map_shared_rank(&sm, warp);
#pragma unroll
      for (int v = 0; v < VEC; ++v) peer->blocks[par][rank][lane][v] = t[v];
    }
    cl.sync();
    float at_block[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) at_block[v] = carry[v];
    for (int r = 0; r < ncl; ++r) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        if (r == rank) at_block[v] = carry[v];
        const float2 m = sm.blocks[par][r][lane][v];
        carry[v] = fmaf(m.x, carry[v], m.y);
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) mine[v] = at_block[v];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w < warp) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float2 r = sm.runs[par][w][lane][v];
          mine[v] = fmaf(r.x, mine[v], r.y);
        }
      }
    }
  } else {
#pragma unroll
    for (int w = 0; w < NW; ++w) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        if (w == warp) mine[v] = carry[v];
        const float2 r = sm.runs[par][w][lane][v];
        carry[v] = fmaf(r.x, carry[v], r.y);
      }
    }
  }
}

template <class T, int VEC, int L, int NW>
__global__ void __launch_bounds__(NW * 32) k_scan_forward(const ScanArgs a) {
  pdl_enter();
  __shared__ Join<VEC, NW> sm;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ncl = a.cluster, rank = ncl > 1 ? (int)(blockIdx.x % ncl) : 0;
  const int unit = blockIdx.x / ncl;
  const int c = ((unit % a.ctiles) * 32 + lane) * VEC;
  const int s = unit / a.ctiles;
  const bool on = c < a.channels;
  int first, len;
  sequence_range(a, s, first, len);
  const int64_t at0 = a.reverse ? (int64_t)first + len - 1 : first;   // the scan's first token
  const int64_t dir = a.reverse ? -1 : 1;
  const T* z = static_cast<const T*>(a.z) + at0 * a.ld_z + c;
  const T* x = static_cast<const T*>(a.x) + at0 * a.ld_x + c;
  T* h = static_cast<T*>(a.h) + at0 * a.ld_h + c;
  const int64_t dz = dir * a.ld_z, dx = dir * a.ld_x, dh = dir * a.ld_h;

  float carry[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    carry[v] = on && a.h0 ? a.h0[(int64_t)s * a.channels + c + v] : 0.0f;
  if (len == 0) {   // (the same for all blocks of the cluster)
    if (a.h_last && on && rank == 0 && warp == 0)
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.h_last[(int64_t)s * a.channels + c + v] = carry[v];
    return;
  }
  if (ncl > 1) cg::this_cluster().sync();   // every block runs before anyone writes to its memory

  const int mine0 = (rank * NW + warp) * L, step = ncl * NW * L;
  uint32_t wz[L], wx[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int t = mine0 + i;
    wz[i] = wx[i] = 0;
    if (on && t < len) {
      wz[i] = load_word<T, VEC>(z + t * dz);
      wx[i] = load_word<T, VEC>(x + t * dx);
    }
  }
  int par = 0;
  for (int64_t base = 0; base < len; base += step, par ^= 1) {
    const int t0 = (int)base + mine0;
    float f[L][VEC], b[L][VEC], P[VEC], S[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) { P[v] = 1.0f; S[v] = 0.0f; }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float zz[VEC], xx[VEC];
      unpack<T, VEC>(wz[i], zz);
      unpack<T, VEC>(wx[i], xx);
      const bool live = t0 + i < len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float omf;
        gate(zz[v], f[i][v], omf);
        b[i][v] = omf * xx[v];
        if (!live) { f[i][v] = 1.0f; b[i][v] = 0.0f; }
        P[v] *= f[i][v];
        S[v] = fmaf(f[i][v], S[v], b[i][v]);
      }
    }
#pragma unroll
    for (int i = 0; i < L; ++i) {   // the next steps' words, under way during the join
      const int64_t t = base + step + mine0 + i;
      if (on && t < len) {
        wz[i] = load_word<T, VEC>(z + t * dz);
        wx[i] = load_word<T, VEC>(x + t * dx);
      }
    }
    float cur[VEC];
    join_runs<VEC, NW>(sm, par, ncl, rank, warp, lane, P, S, carry, cur);
#pragma unroll
    for (int i = 0; i < L; ++i) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) cur[v] = fmaf(f[i][v], cur[v], b[i][v]);
      const int t = t0 + i;
      if (on && t < len) store_word<T, VEC>(h + t * dh, pack<T, VEC>(cur));
    }
    if (a.h_last && on && t0 < len && t0 + L >= len) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.h_last[(int64_t)s * a.channels + c + v] = cur[v];
    }
  }
}

// Backward, walked from the sequence's end: position u = len-1-t.  A thread's run of L steps
// needs h_{t-1} at each of them; it reads the stored h once, before the run's first step, and
// recomputes the others in 32 bits from z and x, which it has to read anyway: 5 words moved a
// step instead of 6, and the states inside a run carry no rounding of the output type.
template <class T, int VEC, int L, int NW>
__global__ void __launch_bounds__(NW * 32) k_scan_backward(const ScanArgs a) {
  pdl_enter();
  __shared__ Join<VEC, NW> sm;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ncl = a.cluster, rank = ncl > 1 ? (int)(blockIdx.x % ncl) : 0;
  const int unit = blockIdx.x / ncl;
  const int c = ((unit % a.ctiles) * 32 + lane) * VEC;
  const int s = unit / a.ctiles;
  const bool on = c < a.channels;
  int first, len;
  sequence_range(a, s, first, len);
  const int64_t at0 = a.reverse ? (int64_t)first + len - 1 : first;
  const int64_t dir = a.reverse ? -1 : 1;
  const T* z = static_cast<const T*>(a.z) + at0 * a.ld_z + c;
  const T* x = static_cast<const T*>(a.x) + at0 * a.ld_x + c;
  const T* h = static_cast<const T*>(a.h_in) + at0 * a.ld_h + c;
  const T* dh = static_cast<const T*>(a.dh) + at0 * a.ld_dh + c;
  T* gz = static_cast<T*>(a.dz) + at0 * a.ld_dz + c;
  T* gx = static_cast<T*>(a.dx) + at0 * a.ld_dx + c;
  const int64_t sz = dir * a.ld_z, sx = dir * a.ld_x, sh = dir * a.ld_h, sdh = dir * a.ld_dh,
                sgz = dir * a.ld_dz, sgx = dir * a.ld_dx;

  float carry[VEC], start[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    carry[v] = on && a.dh_last ? a.dh_last[(int64_t)s * a.channels + c + v] : 0.0f;
    start[v] = on && a.h0 ? a.h0[(int64_t)s * a.channels + c + v] : 0.0f;
  }
  if (len == 0) {
    if (a.dh0 && on && rank == 0 && warp == 0)
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.dh0[(int64_t)s * a.channels + c + v] = carry[v];
    return;
  }
  if (ncl > 1) cg::this_cluster().sync();

  const int mine0 = (rank * NW + warp) * L, step = ncl * NW * L;
  uint32_t wz[L], wx[L], wd[L], wh = 0;
  auto load = [&](int64_t u0) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int64_t t = len - 1 - (u0 + i);
      wz[i] = wx[i] = wd[i] = 0;
      if (on && t >= 0) {
        wz[i] = load_word<T, VEC>(z + t * sz);
        wx[i] = load_word<T, VEC>(x + t * sx);
        wd[i] = load_word<T, VEC>(dh + t * sdh);
      }
    }
    const int64_t before = len - 1 - (u0 + L);   // the step before the run's first
    if (on && before >= 0) wh = load_word<T, VEC>(h + before * sh);
  };
  load(mine0);
  int par = 0;
  for (int64_t base = 0; base < len; base += step, par ^= 1) {
    const int64_t u0 = base + mine0;
    const int64_t t_hi = len - 1 - u0;   // may be negative: nothing of this sequence is left
    float f[L][VEC], w1[L][VEC], d[L][VEC], g[L][VEC], P[VEC], S[VEC], hp[VEC];
    unpack<T, VEC>(wh, hp);
    if (t_hi - L < 0) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) hp[v] = start[v];
    }
#pragma unroll
    for (int i = L - 1; i >= 0; --i) {   // ascending t
      float zz[VEC], xx[VEC];
      unpack<T, VEC>(wz[i], zz);
      unpack<T, VEC>(wx[i], xx);
      unpack<T, VEC>(wd[i], g[i]);
      const bool live = t_hi - i >= 0;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        gate(zz[v], f[i][v], w1[i][v]);
        d[i][v] = hp[v] - xx[v];
        if (live) hp[v] = fmaf(f[i][v], hp[v], w1[i][v] * xx[v]);
        else f[i][v] = 1.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) { P[v] = 1.0f; S[v] = 0.0f; }
#pragma unroll
    for (int i = 0; i < L; ++i) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        P[v] *= f[i][v];
        S[v] = f[i][v] * (g[i][v] + S[v]);
      }
    }
    load(base + step + mine0);
    float cur[VEC];
    join_runs<VEC, NW>(sm, par, ncl, rank, warp, lane, P, S, carry, cur);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float oz[VEC], ox[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float gt = g[i][v] + cur[v];
        cur[v] = f[i][v] * gt;
        ox[v] = w1[i][v] * gt;
        oz[v] = w1[i][v] * cur[v] * d[i][v];
      }
      const int64_t t = t_hi - i;
      if (on && t >= 0) {
        store_word<T, VEC>(gz + t * sgz, pack<T, VEC>(oz));
        store_word<T, VEC>(gx + t * sgx, pack<T, VEC>(ox));
      }
    }
    // (steps before the sequence's first have f = 1, g = 0: they pass e on unchanged)
    if (a.dh0 && on && t_hi >= 0 && t_hi < L) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.dh0[(int64_t)s * a.channels + c + v] = cur[v];
    }
  }
}

// One token a sequence: the state is read, advanced and written back where it lies.
template <class T, int VEC>
__global__ void __launch_bounds__(256)
k_scan_step(const T* z, int64_t ld_z, const T* x, int64_t ld_x, float* state, const int32_t* slots,
            int32_t num_slots, T* out, int64_t ld_out, int32_t rows, int32_t channels) {
  pdl_enter();
  const int words = (channels + VEC - 1) / VEC;
  const int64_t total = (int64_t)rows * words;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int r = (int)(i / words), c = (int)(i % words) * VEC;
    const int slot = slots ? __ldg(slots + r) : r;
    float zz[VEC], xx[VEC], y[VEC];
    unpack<T, VEC>(load_word<T, VEC>(z + r * ld_z + c), zz);
    unpack<T, VEC>(load_word<T, VEC>(x + r * ld_x + c), xx);
    const bool live = slot >= 0 && slot < num_slots;
    float* st = state + (int64_t)(live ? slot : 0) * channels + c;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float f, omf;
      gate(zz[v], f, omf);
      y[v] = live ? fmaf(f, st[v], omf * xx[v]) : 0.0f;
      if (live) st[v] = y[v];
    }
    store_word<T, VEC>(out + r * ld_out + c, pack<T, VEC>(y));
  }
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int kFwdL = 16, kFwdNW = 8, kBwdL = 8, kBwdNW = 16;

int cluster_for(const ScanArgs& a, int tile) {
  int64_t blocks = (int64_t)a.ctiles * a.seqs;
  const int64_t len = a.tokens / std::max(a.seqs, 1);
  int ncl = 1;
  while (ncl < kMaxCluster && blocks * ncl < 296 && (int64_t)ncl * tile < len) ncl *= 2;
  return ncl;
}

template <class T, int VEC>
int32_t enqueue(ScanArgs a, bool backward, cudaStream_t s) {
  a.ctiles = (a.channels + 32 * VEC - 1) / (32 * VEC);
  a.cluster = cluster_for(a, backward ? kBwdL * kBwdNW : kFwdL * kFwdNW);
  const int64_t grid = (int64_t)a.ctiles * a.seqs * a.cluster;
  if (grid > INT32_MAX) return DGC_EINVAL;
  if (backward)
    launch_cluster(k_scan_backward<T, VEC, kBwdL, kBwdNW>, dim3((unsigned)grid), dim3(kBwdNW * 32), 0, s,
                   (unsigned)a.cluster, a);
  else
    launch_cluster(k_scan_forward<T, VEC, kFwdL, kFwdNW>, dim3((unsigned)grid), dim3(kFwdNW * 32), 0, s,
                   (unsigned)a.cluster, a);
  return check_launch();
}

int32_t dispatch(const ScanArgs& a, int32_t dtype, bool backward, bool pairs, cudaStream_t s) {
  if (dtype == DGC_F32) return enqueue<float, 1>(a, backward, s);
  if (dtype == DGC_BF16)
    return pairs ? enqueue<__nv_bfloat16, 2>(a, backward, s) : enqueue<__nv_bfloat16, 1>(a, backward, s);
  return pairs ? enqueue<__half, 2>(a, backward, s) : enqueue<__half, 1>(a, backward, s);
}

size_t element_size(int32_t dtype) { return dtype == DGC_F32 ? 4 : 2; }

bool bad_shape(int32_t dtype, int64_t tokens, int32_t seqs, int32_t channels, const int32_t* seq_start) {
  if (dtype < DGC_F32 || dtype > DGC_F16) return true;
  if (tokens < 0 || tokens > INT32_MAX || seqs < 1 || channels < 1) return true;
  return !seq_start && tokens % seqs != 0;
}

// A matrix argument: rows of `channels` elements, `ld` apart.
bool bad_rows(const void* p, int64_t ld, int32_t channels, size_t elem, int64_t tokens) {
  return ld < channels || (tokens > 0 && (!p || !aligned(p, elem)));
}

bool pairs_ok(const void* p, int64_t ld) { return aligned(p, 4) && ld % 2 == 0; }

}  // namespace

extern "C" {

int32_t dgc_gated_scan_forward(int32_t dtype, int64_t tokens, int32_t num_seqs, int32_t channels,
                               const int32_t* seq_start, int32_t reverse, const void* gate_logits,
                               int64_t ld_gate, const void* x, int64_t ld_x, const float* h0, void* h,
                               int64_t ld_h, float* h_last, void* stream) {
  if (bad_shape(dtype, tokens, num_seqs, channels, seq_start)) return DGC_EINVAL;
  const size_t es = element_size(dtype);
  if (bad_rows(gate_logits, ld_gate, channels, es, tokens) || bad_rows(x, ld_x, channels, es, tokens) ||
      bad_rows(h, ld_h, channels, es, tokens) || !aligned(h0, 4) || !aligned(h_last, 4) ||
      !aligned(seq_start, 4))
    return DGC_EINVAL;
  if (tokens == 0 && !h_last) return DGC_OK;
  ScanArgs a{};
  a.z = gate_logits; a.x = x; a.h = h; a.h0 = h0; a.h_last = h_last; a.seq_start = seq_start;
  a.ld_z = ld_gate; a.ld_x = ld_x; a.ld_h = ld_h;
  a.tokens = (int32_t)tokens; a.seqs = num_seqs; a.seq_len = (int32_t)(tokens / num_seqs);
  a.channels = channels; a.reverse = reverse != 0;
  const bool pairs = channels % 2 == 0 && pairs_ok(gate_logits, ld_gate) && pairs_ok(x, ld_x) && pairs_ok(h, ld_h);
  return dispatch(a, dtype, false, pairs, as_stream(stream));
}

int32_t dgc_gated_scan_backward(int32_t dtype, int64_t tokens, int32_t num_seqs, int32_t channels,
                                const int32_t* seq_start, int32_t reverse, const void* gate_logits,
                                int64_t ld_gate, const void* x, int64_t ld_x, const float* h0,
                                const void* h, int64_t ld_h, const void* dh, int64_t ld_dh,
                                const float* dh_last, void* dgate, int64_t ld_dgate, void* dx,
                                int64_t ld_dx, float* dh0, void* stream) {
  if (bad_shape(dtype, tokens, num_seqs, channels, seq_start)) return DGC_EINVAL;
  const size_t es = element_size(dtype);
  if (bad_rows(gate_logits, ld_gate, channels, es, tokens) || bad_rows(x, ld_x, channels, es, tokens) ||
      bad_rows(h, ld_h, channels, es, tokens) || bad_rows(dh, ld_dh, channels, es, tokens) ||
      bad_rows(dgate, ld_dgate, channels, es, tokens) || bad_rows(dx, ld_dx, channels, es, tokens) ||
      !aligned(h0, 4) || !aligned(dh_last, 4) || !aligned(dh0, 4) || !aligned(seq_start, 4))
    return DGC_EINVAL;
  if (tokens == 0 && !dh0) return DGC_OK;
  ScanArgs a{};
  a.z = gate_logits; a.x = x; a.h_in = h; a.dh = dh; a.dz = dgate; a.dx = dx; a.h0 = h0;
  a.dh_last = dh_last; a.dh0 = dh0; a.seq_start = seq_start;
  a.ld_z = ld_gate; a.ld_x = ld_x; a.ld_h = ld_h; a.ld_dh = ld_dh; a.ld_dz = ld_dgate; a.ld_dx = ld_dx;
  a.tokens = (int32_t)tokens; a.seqs = num_seqs; a.seq_len = (int32_t)(tokens / num_seqs);
  a.channels = channels; a.reverse = reverse != 0;
  const bool pairs = channels % 2 == 0 && pairs_ok(gate_logits, ld_gate) && pairs_ok(x, ld_x) &&
                     pairs_ok(h, ld_h) && pairs_ok(dh, ld_dh) && pairs_ok(dgate, ld_dgate) && pairs_ok(dx, ld_dx);
  return dispatch(a, dtype, true, pairs, as_stream(stream));
}

int32_t dgc_gated_scan_step(int32_t dtype, int32_t rows, int32_t channels, const void* gate_logits,
                            int64_t ld_gate, const void* x, int64_t ld_x, float* state,
                            const int32_t* slots, int32_t num_slots, void* out, int64_t ld_out,
                            void* stream) {
  if (dtype < DGC_F32 || dtype > DGC_F16 || rows < 0 || channels < 1 || num_slots < 0) return DGC_EINVAL;
  const size_t es = element_size(dtype);
  if (bad_rows(gate_logits, ld_gate, channels, es, rows) || bad_rows(x, ld_x, channels, es, rows) ||
      bad_rows(out, ld_out, channels, es, rows) || !aligned(slots, 4))
    return DGC_EINVAL;
  if (rows == 0) return DGC_OK;
  if (!state || !aligned(state, 4) || (!slots && num_slots < rows)) return DGC_EINVAL;
  cudaStream_t s = as_stream(stream);
  const bool pairs = channels % 2 == 0 && pairs_ok(gate_logits, ld_gate) && pairs_ok(x, ld_x) && pairs_ok(out, ld_out);
  auto go = [&](auto tag, auto vec) {
    using T = decltype(tag);
    constexpr int VEC = decltype(vec)::value;
    const int64_t total = (int64_t)rows * (channels / VEC);
    const int grid = (int)std::min<int64_t>((total + 255) / 256, 148 * 8);
    launch(k_scan_step<T, VEC>, grid, 256, 0, s, static_cast<const T*>(gate_logits), ld_gate,
           static_cast<const T*>(x), ld_x, state, slots, num_slots, static_cast<T*>(out), ld_out, rows, channels);
  };
  using one = std::integral_constant<int, 1>;
  using two = std::integral_constant<int, 2>;
  if (dtype == DGC_F32) go(float{}, one{});
  else if (dtype == DGC_BF16) pairs ? go(__nv_bfloat16{}, two{}) : go(__nv_bfloat16{}, one{});
  else pairs ? go(__half{}, two{}) : go(__half{}, one{});
  return check_launch();
}

}  // extern "C"
