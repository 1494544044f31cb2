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
// consecutive steps of 32 such words.  A block of NW warps holds NW*L steps; a cluster of blocks
// holds consecutive ones.  Every warp fetches its own rows into shared memory with 16-byte
// asynchronous copies, a stage ahead, whatever the alignment of the rows (see copy_rows).  Every
// thread walks its run once to reduce it to (P, S), the runs are joined in order through shared
// memory (the blocks' through the cluster's), and a second walk over the coefficients kept in
// registers starts from the true state.  One pass over the data, no workspace, and a fixed
// order of the additions: results do not vary from run to run.
//
// A sequence is one cluster's work, so nothing (no infinity, no NaN) can cross from one
// sequence into its neighbour in the pack.

#include <cooperative_groups.h>

#include <algorithm>
#include <cstdlib>
#include <initializer_list>

#include "common.cuh"

namespace cg = cooperative_groups;
using namespace dgc;

namespace {

constexpr int kMaxCluster = 8;
constexpr unsigned long long kWaitNs = 1000000000ull;   // bound of a wait on a peer: a second

// A matrix argument.  The strides that the loops add are laid out by the host: as kernel
// parameters they cost no registers.
struct Matrix {
  char *begin, *end;
  int64_t ld;        // elements
  int64_t stride;    // bytes from one step of the walk to the next (negative: towards the front)
  int64_t jump;      // stride * steps of a round
  int64_t skip;      // stride * (steps of a round - steps of a run)
};

struct ScanArgs {
  Matrix z, x, h, dh, dz, dx;
  const float *h0, *dh_last;
  float *h_last, *dh0;
  const int32_t* seq_start;
  int32_t tokens, seqs, seq_len, channels, ctiles, cluster, reverse;
};

// The channels of a lane's word, with the packed 32-bit arithmetic of sm_100 (two operations an
// instruction, each rounded as its scalar form).
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

// f = sigma(z) and 1 - f, each to full relative precision (1 - f is not formed by subtraction:
// for gates near 1 it is the weight of the input).  The logit is held above -87, so that e f
// cannot become inf * 0; f is then at most 2e-38 too large.  A NaN passes through.
template <int VEC>
__device__ __forceinline__ void gate(Val<VEC> z, Val<VEC>& f, Val<VEC>& omf) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) asm("max.NaN.f32 %0, %0, 0fC2AE0000;" : "+f"(z.v[i]));   // -87
  const Val<VEC> x = mul_(z, fill<VEC>(-1.4426950408889634f));
  Val<VEC> e;
#pragma unroll
  for (int i = 0; i < VEC; ++i) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.v[i]) : "f"(x.v[i]));
  const Val<VEC> t = add_(e, fill<VEC>(1.0f));
#pragma unroll
  for (int i = 0; i < VEC; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f.v[i]) : "f"(t.v[i]));
  omf = mul_(e, f);
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

// ------------------------------------------------------------------ joining the runs
// A map y_out = P y_in + S of a lane's channels, as it lies in shared memory.
template <int VEC> struct alignas(8 * VEC) Map { Val<VEC> p, s; };

// The maps of a block's runs, the states they start from, and the maps of the cluster's blocks.
// Everything alternates between two buffers from round to round.
template <int VEC, int NW>
struct Join {
  Map<VEC> runs[2][NW][32];
  Map<VEC> blocks[2][kMaxCluster][32];
  Val<VEC> starts[2][NW][32];
  unsigned long long arrived[2];             // mbarriers of `blocks`
};

// Waits that run out (they cannot, short of a fault: the blocks of a cluster run together) are
// counted here and not waited for again; dgc_gated_scan_check reports them.
__device__ int g_scan_waits_out;

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

template <int VEC, int NW>
__device__ __forceinline__ void join_begin(Join<VEC, NW>& sm, int ncl) {
  if (ncl == 1) return;
  if (threadIdx.x < 2)
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&sm.arrived[threadIdx.x])) : "memory");
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  cg::this_cluster().sync();   // every block runs, its barriers are there
}

__device__ __forceinline__ unsigned long long clock_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}

__device__ __forceinline__ bool wait_arrived(uint32_t barrier, uint32_t phase) {
  unsigned long long since = 0;
  for (;;) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(barrier), "r"(phase) : "memory");
    if (done) return true;
    if (since == 0) since = clock_ns();
    else if (clock_ns() - since > kWaitNs) break;
  }
  atomicAdd(&g_scan_waits_out, 1);
  return false;
}

// Joins the runs of all warps of the cluster in order: takes this warp's map (P, S), returns the
// state its run starts from.  The first warp does the work for the block; it alone holds
// `carry`, the state before the cluster's first run on entry and after its last on return.
// A block's map reaches the others by asynchronous stores that complete on their barriers, not
// through the cluster's barrier: that one would wait for every store of results under way.
template <int VEC, int NW>
__device__ __forceinline__ Val<VEC> join_runs(Join<VEC, NW>& sm, int round, int ncl, int rank, int warp, int lane,
                                              const Val<VEC>& P, const Val<VEC>& S, Val<VEC>& carry, bool& waits) {
  const int par = round & 1;
  sm.runs[par][warp][lane] = {P, S};
  __syncthreads();
  if (warp == 0) {
    Val<VEC> cur = carry;
    if (ncl > 1) {
      Val<VEC> tp = P, ts = S;
#pragma unroll
      for (int w = 1; w < NW; ++w) {
        const Map<VEC> m = sm.runs[par][w][lane];
        tp = mul_(m.p, tp);
        ts = fma_(m.p, ts, m.s);
      }
      const uint32_t to = shared_address(&sm.blocks[par][rank][lane]), bar = shared_address(&sm.arrived[par]);
      if (lane == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(ncl * 32 * 2 * VEC * 4) : "memory");
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        if (r < ncl) {
          uint32_t far, far_bar;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(to), "r"(r));
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far_bar) : "r"(bar), "r"(r));
          if constexpr (VEC == 2)
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                         ::"r"(far), "f"(tp.v[0]), "f"(tp.v[1]), "f"(ts.v[0]), "f"(ts.v[1]), "r"(far_bar) : "memory");
          else
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                         ::"r"(far), "f"(tp.v[0]), "f"(ts.v[0]), "r"(far_bar) : "memory");
        }
      }
      if (waits) waits = wait_arrived(bar, (uint32_t)(round >> 1) & 1u);
#pragma unroll
      for (int r0 = 0; r0 < kMaxCluster; r0 += 4) {   // (four loads under way at a time)
        if (r0 < ncl) {
          Map<VEC> m[4];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (r0 + r < ncl) m[r] = sm.blocks[par][r0 + r][lane];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (r0 + r == rank) cur = carry;
            if (r0 + r < ncl) carry = fma_(m[r].p, carry, m[r].s);
          }
        }
      }
    }
#pragma unroll
    for (int w0 = 0; w0 < NW; w0 += 4) {
      Map<VEC> m[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) m[w] = sm.runs[par][w0 + w][lane];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        sm.starts[par][w0 + w][lane] = cur;
        cur = fma_(m[w].p, cur, m[w].s);
      }
    }
    if (ncl == 1) carry = cur;
  }
  __syncthreads();
  return sm.starts[par][warp][lane];
}

// ------------------------------------------------------------------ rows into shared memory
// How the rows lie against 16-byte boundaries, over all matrices of a call.
enum Lie { kAligned, kWords, kHalves };   // every row on a boundary; on 4 bytes; on 2 bytes

constexpr int kRowBytes = 128;            // a warp's part of a row: 32 words
template <Lie LIE> constexpr int kGranules = LIE == kAligned ? kRowBytes / 16 : kRowBytes / 16 + 1;
template <Lie LIE> constexpr int kPitch = kGranules<LIE> * 16;

// Where a matrix's row `row` has this block's channels.
template <class T>
__device__ __forceinline__ char* row_at(const Matrix& m, int64_t row, int c) {
  return m.begin + (row * m.ld + c) * (int64_t)sizeof(T);
}

// Copies the warp's part of the rows [lo, hi) of a round's L, from `next` on, and moves `next` on
// by a round; `width` is the part's bytes inside the matrix's columns.  (Where rows are aligned
// `next` is this lane's granule.)  Where rows do not start on a boundary the granules at a
// part's ends also hold neighbouring elements, which nobody uses; a granule that reaches
// outside the matrix itself is fetched by elements.
template <class T, Lie LIE, int L>
__device__ __forceinline__ void copy_rows(char* to, const char*& next, const Matrix& m, int64_t stride, int64_t jump,
                                          int lo, int hi, int width, int lane) {
  constexpr int G = kGranules<LIE>;
  if constexpr (LIE == kAligned) {
    static_assert(G == 8 && L % 4 == 0, "");
    const int r0 = lane / 8, g = lane % 8;
    const uint32_t dst = shared_address(to) + r0 * kPitch<LIE> + g * 16;
    const char* p = next;
    if (g * 16 >= width) hi = 0;
#pragma unroll
    for (int k = 0; k < L / 4; ++k, p += 4 * stride)
      if (r0 + 4 * k >= lo && r0 + 4 * k < hi)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 4 * k * kPitch<LIE>), "l"(p) : "memory");
  } else {
    const uint32_t dst = shared_address(to);
#pragma unroll
    for (int k = 0; k < (L * G + 31) / 32; ++k) {
      const int i = lane + 32 * k, r = i / G, g = i % G;
      if (r >= lo && r < hi) {
        const char* p = next + r * stride;
        const char* q = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15) + g * 16;
        if (q < p + width) {
          if (q >= m.begin && q + 16 <= m.end) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + r * kPitch<LIE> + g * 16), "l"(q)
                         : "memory");
          } else {
            for (int b = 0; b < 16; b += sizeof(T))
              if (q + b >= p && q + b < p + width)
                *reinterpret_cast<T*>(to + r * kPitch<LIE> + g * 16 + b) = *reinterpret_cast<const T*>(q + b);
          }
        }
      }
    }
  }
  next += jump;
}

// Where a lane's copies of a round start.
template <class T, Lie LIE>
__device__ __forceinline__ const char* first_copy(const Matrix& m, int64_t row, int c0, int64_t stride, int lane) {
  const char* p = row_at<T>(m, row, c0);
  return LIE == kAligned ? p + (lane / 8) * stride + lane % 8 * 16 : p;
}

// Word of this lane in row r of a copied part; `first` is the low half of the address of the
// part's first row, `stride` the low half of the stride.
template <class T, Lie LIE>
__device__ __forceinline__ Val<4 / sizeof(T)> row_word(const char* from, uint32_t first, uint32_t stride, int r,
                                                       int lane) {
  Val<4 / sizeof(T)> w;
  const char* p = from + r * kPitch<LIE> + lane * 4;
  if (LIE != kAligned) p += (first + r * stride) & 15u;
  if constexpr (LIE == kHalves) {
    static_assert(sizeof(T) == 2, "");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float one[1];
      unpack<T, 1>(*reinterpret_cast<const unsigned short*>(p + 2 * i), one);
      w.v[i] = one[0];
    }
  } else {
    unpack<T, 4 / sizeof(T)>(*reinterpret_cast<const uint32_t*>(p), w.v);
  }
  return w;
}

template <class T, Lie LIE>
__device__ __forceinline__ void put_word(char* p, const Val<4 / sizeof(T)>& w, bool on0, bool on1) {
  if constexpr (LIE == kHalves) {
    const float a[1] = {w.v[0]}, b[1] = {w.v[1]};
    if (on0) store_word<T, 1>(reinterpret_cast<T*>(p), pack<T, 1>(a));
    if (on1) store_word<T, 1>(reinterpret_cast<T*>(p) + 1, pack<T, 1>(b));
  } else {
    if (on0) store_word<T, 4 / sizeof(T)>(reinterpret_cast<T*>(p), pack<T, 4 / sizeof(T)>(w.v));
  }
}

template <int N>
__device__ __forceinline__ void wait_copies() {   // all but the last N groups have arrived
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
  __syncwarp();
}
__device__ __forceinline__ void end_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// What a thread works on: a sequence, a block of channels, a place in the cluster.
template <class T, int L, int NW>
struct Place {
  static constexpr int VEC = 4 / sizeof(T);
  int lane, warp, ncl, rank, s, c0, c, first, len, mine0, step, width;
  bool on0, on1;
  int64_t at0, dir;
  __device__ __forceinline__ explicit Place(const ScanArgs& a) {
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    ncl = a.cluster;
    rank = ncl > 1 ? (int)(blockIdx.x % ncl) : 0;
    const int unit = blockIdx.x / ncl;
    s = unit / a.ctiles;
    c0 = (unit % a.ctiles) * 32 * VEC;
    c = c0 + lane * VEC;
    on0 = c < a.channels;
    on1 = c + 1 < a.channels;
    width = min(32 * VEC, a.channels - c0) * (int)sizeof(T);
    sequence_range(a, s, first, len);
    at0 = a.reverse ? (int64_t)first + len - 1 : first;   // the scan's first token
    dir = a.reverse ? -1 : 1;
    mine0 = (rank * NW + warp) * L;
    step = ncl * NW * L;
  }
  __device__ __forceinline__ Val<VEC> get(const float* p, int channels) const {
    Val<VEC> w;
#pragma unroll
    for (int i = 0; i < VEC; ++i) w.v[i] = p && (i ? on1 : on0) ? p[(int64_t)s * channels + c + i] : 0.0f;
    return w;
  }
  __device__ __forceinline__ void put(float* p, int channels, const Val<VEC>& w) const {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i ? on1 : on0) p[(int64_t)s * channels + c + i] = w.v[i];
  }
};

constexpr int kStages = 2;

template <class T, Lie LIE, int L, int NW, int BLOCKS>
__global__ void __launch_bounds__(NW * 32, BLOCKS) k_scan_forward(const ScanArgs a) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), kPart = L * kPitch<LIE>;
  extern __shared__ __align__(16) char buffer[];   // [warp][stage][z, x][L rows]
  __shared__ Join<VEC, NW> sm;
  const Place<T, L, NW> at(a);
  const int len = at.len;
  const int64_t row0 = at.at0 + at.dir * at.mine0;
  const char* z = first_copy<T, LIE>(a.z, row0, at.c0, a.z.stride, at.lane);
  const char* x = first_copy<T, LIE>(a.x, row0, at.c0, a.x.stride, at.lane);
  // (low halves of addresses: where in their granules the rows of the round in hand start)
  uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(z), x0 = (uint32_t)reinterpret_cast<uintptr_t>(x);
  char* const mine = buffer + at.warp * (kStages * 2 * kPart);
  int ahead = len - at.mine0;   // steps from the next fetch's first on (may be negative)
  auto fetch = [&](int stage) {
    copy_rows<T, LIE, L>(mine + stage * 2 * kPart, z, a.z, a.z.stride, a.z.jump, 0, min(ahead, L), at.width, at.lane);
    copy_rows<T, LIE, L>(mine + stage * 2 * kPart + kPart, x, a.x, a.x.stride, a.x.jump, 0, min(ahead, L), at.width, at.lane);
    end_copies();
    ahead = max(ahead - at.step, 0);
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) fetch(i);
  Val<VEC> carry = at.get(a.h0, a.channels);
  if (len == 0) {   // (the same for all blocks of the cluster)
    if (a.h_last && at.rank == 0 && at.warp == 0) at.put(a.h_last, a.channels, carry);
    return;
  }
  join_begin(sm, at.ncl);

  char* out = row_at<T>(a.h, row0, at.c);
  bool waits = true;
  int stage = 0;
  const int rounds = (len - 1) / at.step + 1;
  int left = len - at.mine0;   // steps from this warp's first of the round on
  for (int round = 0; round < rounds; ++round, left -= at.step) {
    const bool full = left >= L;
    const char* from = mine + stage * 2 * kPart;
    Val<VEC> f[L], b[L], P = fill<VEC>(1.0f), S = fill<VEC>(0.0f);
    wait_copies<kStages - 1>();
    auto walk = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        Val<VEC> omf;
        gate(row_word<T, LIE>(from, z0, (uint32_t)a.z.stride, i, at.lane), f[i], omf);
        b[i] = mul_(omf, row_word<T, LIE>(from + kPart, x0, (uint32_t)a.x.stride, i, at.lane));
        if (!decltype(whole)::value && i >= left) { f[i] = fill<VEC>(1.0f); b[i] = fill<VEC>(0.0f); }
        P = mul_(P, f[i]);
        S = fma_(f[i], S, b[i]);
      }
    };
    if (full) walk(std::true_type{});
    else walk(std::false_type{});
    __syncwarp();   // the stage has been read by all lanes
    fetch(stage);
    stage ^= 1;
    z0 += (uint32_t)a.z.jump;
    x0 += (uint32_t)a.x.jump;
    Val<VEC> cur = join_runs<VEC, NW>(sm, round, at.ncl, at.rank, at.warp, at.lane, P, S, carry, waits);
    auto write = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < L; ++i, out += a.h.stride) {
        cur = fma_(f[i], cur, b[i]);
        if (decltype(whole)::value || i < left) put_word<T, LIE>(out, cur, at.on0, at.on1);
      }
    };
    if (full) write(std::true_type{});
    else write(std::false_type{});
    out += a.h.skip;
    // (steps after the last have f = 1, b = 0: they pass the state on unchanged)
    if (a.h_last && left > 0 && left <= L) at.put(a.h_last, a.channels, cur);
  }
  wait_copies<0>();
}

// Backward, walked from the sequence's end: position u = len-1-t.  A thread's run of L steps
// needs h_{t-1} at each of them; it reads the stored h once, before the run's first step, and
// recomputes the others in 32 bits from z and x, which it has to read anyway: 5 words moved a
// step instead of 6, and the states inside a run carry no rounding of the output type.
template <class T, Lie LIE, int L, int NW, int BLOCKS>
__global__ void __launch_bounds__(NW * 32, BLOCKS) k_scan_backward(const ScanArgs a) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), kPart = L * kPitch<LIE>;
  extern __shared__ __align__(16) char buffer[];   // [warp][stage][z, x, dh][L rows]
  __shared__ Join<VEC, NW> sm;
  const Place<T, L, NW> at(a);
  const int len = at.len;
  // a stage holds the steps t_lo .. t_lo + L - 1 in ascending order; the rounds descend
  const int64_t row0 = at.at0 + at.dir * (int64_t)(len - L - at.mine0);
  const char* z = first_copy<T, LIE>(a.z, row0, at.c0, a.z.stride, at.lane);
  const char* x = first_copy<T, LIE>(a.x, row0, at.c0, a.x.stride, at.lane);
  const char* d = first_copy<T, LIE>(a.dh, row0, at.c0, a.dh.stride, at.lane);
  uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(z), x0 = (uint32_t)reinterpret_cast<uintptr_t>(x),
           d0 = (uint32_t)reinterpret_cast<uintptr_t>(d);
  char* const mine = buffer + at.warp * (kStages * 3 * kPart);
  int ahead = len - at.mine0;   // steps of the next fetch and before it (may be negative)
  auto fetch = [&](int stage) {
    char* to = mine + stage * 3 * kPart;
    const int lo = ahead > 0 ? max(L - ahead, 0) : L;
    copy_rows<T, LIE, L>(to, z, a.z, a.z.stride, -a.z.jump, lo, L, at.width, at.lane);
    copy_rows<T, LIE, L>(to + kPart, x, a.x, a.x.stride, -a.x.jump, lo, L, at.width, at.lane);
    copy_rows<T, LIE, L>(to + 2 * kPart, d, a.dh, a.dh.stride, -a.dh.jump, lo, L, at.width, at.lane);
    end_copies();
    ahead = max(ahead - at.step, 0);
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) fetch(i);
  Val<VEC> carry = at.get(a.dh_last, a.channels);
  const Val<VEC> start = at.get(a.h0, a.channels);
  if (len == 0) {
    if (a.dh0 && at.rank == 0 && at.warp == 0) at.put(a.dh0, a.channels, carry);
    return;
  }
  join_begin(sm, at.ncl);

  // the state before a run, stored by the forward pass: fetched a round ahead, as it lies
  uint32_t before[2] = {0, 0};
  auto fetch_state = [&](int left) {
    if (left > L) {
      const T* p = reinterpret_cast<const T*>(row_at<T>(a.h, at.at0 + at.dir * (int64_t)(left - L - 1), at.c));
      if constexpr (LIE == kHalves) {
        if (at.on0) before[0] = load_word<T, 1>(p);
        if (at.on1) before[1] = load_word<T, 1>(p + 1);
      } else {
        if (at.on0) before[0] = load_word<T, VEC>(p);
      }
    }
  };
  int left = len - at.mine0;   // steps up to this warp's last of the round (t_hi + 1)
  char* gz = row_at<T>(a.dz, at.at0 + at.dir * (int64_t)(left - 1), at.c);
  char* gx = row_at<T>(a.dx, at.at0 + at.dir * (int64_t)(left - 1), at.c);
  fetch_state(left);
  bool waits = true;
  int stage = 0;
  const int rounds = (len - 1) / at.step + 1;
  for (int round = 0; round < rounds; ++round, left -= at.step) {
    const bool full = left >= L;
    const int none = L - left;   // steps j of the run below this are before the sequence's first
    const char* from = mine + stage * 3 * kPart;
    Val<VEC> f[L], w[L], e[L], P = fill<VEC>(1.0f), S = fill<VEC>(0.0f);   // f, 1 - f, h_{t-1} - x_t
    Val<VEC> hp;
    if constexpr (LIE == kHalves) {
      unpack<T, 2>(before[0] | before[1] << 16, hp.v);
    } else {
      unpack<T, VEC>(before[0], hp.v);
    }
    if (left <= L) hp = start;
    wait_copies<kStages - 1>();
    auto walk = [&](auto whole) {
#pragma unroll
      for (int j = 0; j < L; ++j) {
        gate(row_word<T, LIE>(from, z0, (uint32_t)a.z.stride, j, at.lane), f[j], w[j]);
        const Val<VEC> x_t = row_word<T, LIE>(from + kPart, x0, (uint32_t)a.x.stride, j, at.lane);
        e[j] = sub_(hp, x_t);
        if (decltype(whole)::value || j >= none) hp = fma_(f[j], hp, mul_(w[j], x_t));
        else f[j] = fill<VEC>(1.0f);
      }
#pragma unroll
      for (int j = L - 1; j >= 0; --j) {
        Val<VEC> g = row_word<T, LIE>(from + 2 * kPart, d0, (uint32_t)a.dh.stride, j, at.lane);
        if (!decltype(whole)::value && j < none) g = fill<VEC>(0.0f);
        P = mul_(P, f[j]);
        S = mul_(f[j], add_(g, S));
      }
    };
    if (full) walk(std::true_type{});
    else walk(std::false_type{});
    fetch_state(left - at.step);
    Val<VEC> cur = join_runs<VEC, NW>(sm, round, at.ncl, at.rank, at.warp, at.lane, P, S, carry, waits);
    auto write = [&](auto whole) {
#pragma unroll
      for (int j = L - 1; j >= 0; --j, gz -= a.dz.stride, gx -= a.dx.stride) {
        if (decltype(whole)::value || j >= none) {
          const Val<VEC> gt = add_(row_word<T, LIE>(from + 2 * kPart, d0, (uint32_t)a.dh.stride, j, at.lane), cur);
          cur = mul_(f[j], gt);
          put_word<T, LIE>(gx, mul_(w[j], gt), at.on0, at.on1);
          put_word<T, LIE>(gz, mul_(mul_(w[j], cur), e[j]), at.on0, at.on1);
        }
      }
    };
    if (full) write(std::true_type{});
    else write(std::false_type{});
    gz -= a.dz.skip;
    gx -= a.dx.skip;
    if (a.dh0 && left > 0 && left <= L) at.put(a.dh0, a.channels, cur);
    __syncwarp();   // the stage has been read by all lanes
    fetch(stage);
    stage ^= 1;
    z0 -= (uint32_t)a.z.jump;
    x0 -= (uint32_t)a.x.jump;
    d0 -= (uint32_t)a.dh.jump;
  }
  wait_copies<0>();
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
    Val<VEC> zz, xx, f, omf;
    float y[VEC];
    unpack<T, VEC>(load_word<T, VEC>(z + r * ld_z + c), zz.v);
    unpack<T, VEC>(load_word<T, VEC>(x + r * ld_x + c), xx.v);
    gate(zz, f, omf);
    const bool live = slot >= 0 && slot < num_slots;
    float* st = state + (int64_t)(live ? slot : 0) * channels + c;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      y[v] = live ? fmaf(f.v[v], st[v], omf.v[v] * xx.v[v]) : 0.0f;
      if (live) st[v] = y[v];
    }
    store_word<T, VEC>(out + r * ld_out + c, pack<T, VEC>(y));
  }
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#ifndef FL
#define FL 16
#define FW 8
#define FB 2
#endif
#ifndef BL
#define BL 8
#define BW 8
#define BB 2
#endif
int cluster_for(const ScanArgs& a, int tile) {
  int64_t blocks = (int64_t)a.ctiles * a.seqs;
  const int64_t len = a.tokens / std::max(a.seqs, 1);
  if (getenv("NCL")) return atoi(getenv("NCL"));
  int ncl = 1;
  while (ncl < kMaxCluster && blocks * ncl < 296 && (int64_t)ncl * tile < len) ncl *= 2;
  return ncl;
}

template <class T, Lie LIE>
int32_t enqueue(ScanArgs a, bool backward, cudaStream_t s) {
  constexpr int VEC = 4 / sizeof(T);
  const int L = backward ? BL : FL, NW = backward ? BW : FW;
  a.ctiles = (a.channels + 32 * VEC - 1) / (32 * VEC);
  a.cluster = cluster_for(a, L * NW);
  const int64_t grid = (int64_t)a.ctiles * a.seqs * a.cluster;
  if (grid > INT32_MAX) return DGC_EINVAL;
  for (Matrix* m : {&a.z, &a.x, &a.h, &a.dh, &a.dz, &a.dx}) {
    m->end = m->begin + ((int64_t)(a.tokens - 1) * m->ld + a.channels) * (int64_t)sizeof(T);
    m->stride = (a.reverse ? -m->ld : m->ld) * (int64_t)sizeof(T);
    m->jump = m->stride * (a.cluster * NW * L);
    m->skip = m->stride * (a.cluster * NW * L - L);
  }
  auto go = [&](auto kernel, size_t smem) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) {
      (void)cudaGetLastError();
      return (int32_t)DGC_ECUDA;
    }
    launch_cluster(kernel, dim3((unsigned)grid), dim3(NW * 32), smem, s, (unsigned)a.cluster, a);
    return check_launch();
  };
  if (backward) return go(k_scan_backward<T, LIE, BL, BW, BB>, NW * kStages * 3 * L * kPitch<LIE>);
  return go(k_scan_forward<T, LIE, FL, FW, FB>, NW * kStages * 2 * L * kPitch<LIE>);
}

int32_t dispatch(const ScanArgs& a, int32_t dtype, bool backward, Lie lie, cudaStream_t s) {
  if (dtype == DGC_F32)
    return lie == kAligned ? enqueue<float, kAligned>(a, backward, s) : enqueue<float, kWords>(a, backward, s);
  if (dtype == DGC_BF16)
    return lie == kAligned ? enqueue<__nv_bfloat16, kAligned>(a, backward, s)
           : lie == kWords ? enqueue<__nv_bfloat16, kWords>(a, backward, s)
                           : enqueue<__nv_bfloat16, kHalves>(a, backward, s);
  return lie == kAligned ? enqueue<__half, kAligned>(a, backward, s)
         : lie == kWords ? enqueue<__half, kWords>(a, backward, s)
                         : enqueue<__half, kHalves>(a, backward, s);
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

Matrix matrix(const void* p, int64_t ld) {
  Matrix m{};
  m.begin = static_cast<char*>(const_cast<void*>(p));
  m.ld = ld;
  return m;
}

// The worst lie of the call's matrices.
Lie lie_of(std::initializer_list<Matrix> ms, int32_t channels, size_t es) {
  size_t bits = channels * es;
  for (const Matrix& m : ms) bits |= reinterpret_cast<uintptr_t>(m.begin) | (size_t)m.ld * es;
  return bits % 16 == 0 ? kAligned : bits % 4 == 0 ? kWords : kHalves;
}

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
  a.z = matrix(gate_logits, ld_gate); a.x = matrix(x, ld_x); a.h = matrix(h, ld_h);
  a.h0 = h0; a.h_last = h_last; a.seq_start = seq_start;
  a.tokens = (int32_t)tokens; a.seqs = num_seqs; a.seq_len = (int32_t)(tokens / num_seqs);
  a.channels = channels; a.reverse = reverse != 0;
  const Lie lie = lie_of({a.z, a.x, a.h}, channels, es);
  return dispatch(a, dtype, false, lie, as_stream(stream));
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
  a.z = matrix(gate_logits, ld_gate); a.x = matrix(x, ld_x); a.h = matrix(h, ld_h);
  a.dh = matrix(dh, ld_dh); a.dz = matrix(dgate, ld_dgate); a.dx = matrix(dx, ld_dx);
  a.h0 = h0; a.dh_last = dh_last; a.dh0 = dh0; a.seq_start = seq_start;
  a.tokens = (int32_t)tokens; a.seqs = num_seqs; a.seq_len = (int32_t)(tokens / num_seqs);
  a.channels = channels; a.reverse = reverse != 0;
  const Lie lie = lie_of({a.z, a.x, a.h, a.dh, a.dz, a.dx}, channels, es);
  return dispatch(a, dtype, true, lie, as_stream(stream));
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

int32_t dgc_gated_scan_check(void* stream) {
  DGC_CUDA(cudaStreamSynchronize(as_stream(stream)));
  int count = 0;
  DGC_CUDA(cudaMemcpyFromSymbol(&count, g_scan_waits_out, sizeof count));
  if (count == 0) return DGC_OK;
  const int none = 0;
  DGC_CUDA(cudaMemcpyToSymbol(g_scan_waits_out, &none, sizeof none));
  return DGC_ECUDA;
}

}  // extern "C"
