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
// registers starts from the true state.  One pass over the data, and a fixed order of the
// additions: results do not vary from run to run.  A few long, narrow sequences go another way,
// by a workspace: see there.
//
// A sequence's runs are joined among themselves alone, so nothing (no infinity, no NaN) can cross from one
// sequence into its neighbour in the pack.

#include <cooperative_groups.h>

#include <algorithm>
#include <initializer_list>

#include "common.cuh"

namespace cg = cooperative_groups;
using namespace dgc;

namespace {

constexpr int kMaxCluster = 16, kPortableCluster = 8;
// Bound of a wait on a peer: a second, of which a time in which nothing of the GPU ran (another
// process's turn, a debugger) counts as a hundredth.
constexpr uint32_t kWaitNs = 1000000000, kPauseNs = kWaitNs / 100;

// A matrix argument.  The strides that the loops add are laid out by the host: as kernel
// parameters they cost no registers.
struct Matrix {
  char *begin, *end;
  int64_t ld;        // elements
  int64_t stride;    // bytes from one step of the walk to the next (negative: towards the front)
};

struct ScanArgs {
  Matrix z, x, h, dh, dz, dx;
  const float *h0, *dh_last;
  float *h_last, *dh0;
  const int32_t* seq_start;
  int32_t tokens, seqs, seq_len, channels, ctiles, cluster, reverse, longest_first;
};

// f = sigma(z) and 1 - f, each within 4.8e-7 + 7.4e-8 |z| of itself: 1 - f is not formed by
// subtraction, for gates near 1 it is the weight of the input.  The term in |z| is the rounding of
// z log2(e) before the exponential (2^-24 |z| of it) and of the constant.  It is left: f and 1 - f
// come from one exponential and move together, so that h sees f (1 - f) of it, and to take it back
// (the product's remainder by a multiply-add, times ln(2), onto the exponential) made calls bound by
// issue 4 to 7 % slower (65536 x 2048 bf16 forward and backward 446 -> 472 us).  The logit is held
// above -87, so that e f cannot become inf * 0; f is then at most 2e-38 too large.  A NaN passes.
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

// The sequence that is `place`-th in length (the longest first, the first first among equals):
// blocks start in this order, so that the last to start have little left to do.
constexpr int kSorted = 128;
__device__ __forceinline__ int by_length(const ScanArgs& a, int place) {
  __shared__ __align__(16) int lens[kSorted];
  __shared__ int found;
  for (int t = threadIdx.x; t < a.seqs; t += blockDim.x) {
    int first;
    sequence_range(a, t, first, lens[t]);
  }
  __syncthreads();
  for (int t = threadIdx.x; t < a.seqs; t += blockDim.x) {
    const int len = lens[t];
    int before = 0;
    for (int j = 0; j < a.seqs; ++j) before += lens[j] > len || (lens[j] == len && j < t);
    if (before == place) found = t;
  }
  __syncthreads();
  return found;
}

// ------------------------------------------------------------------ joining the runs
// A map y_out = P y_in + S of a lane's channels, as it lies in shared memory.
template <int VEC> struct alignas(8 * VEC) Map { Val<VEC> p, s; };

// The product of a run's coefficients, none of which is 0, held at the smallest normal number where
// it underflows: times an infinite y_in it must be infinite, not NaN (a finite one gets at most
// 2^-126 of itself too much).
__device__ __forceinline__ float held(float p) { return fmaxf(p, 0x1p-126f); }
template <int VEC>
__device__ __forceinline__ Val<VEC> held(Val<VEC> p) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) p.v[i] = held(p.v[i]);
  return p;
}

// A block's warps work in G groups that take the rounds in turn.  By group: the maps of a round's
// runs and the states they start from; by round, where there are two groups: the maps of the cluster's
// blocks and the state before the round.  (Slots of `blocks`: a block sends round i + 4 after it has
// every block's map of round i + 2, and the warp that sent that one has read round i by then.)  Only
// blocks of two groups stand in clusters.
constexpr int kBlockSlots = 4;
template <int VEC, int G, int CL>   // CL: the most blocks of a cluster
struct Exchange {
  Map<VEC> blocks[kBlockSlots][CL][32];
  Val<VEC> carry[2][32];
  unsigned long long arrived[kBlockSlots];   // mbarriers of `blocks`
  int gone[G];                               // a wait of the group's ran out
};
template <int VEC>
struct Exchange<VEC, 1, 1> {};
template <int VEC, int NW, int G, int CL>
struct Join : Exchange<VEC, G, CL> {
  static_assert((G == 2) == (CL > 1), "");
  Map<VEC> runs[G][NW][32];
  Val<VEC> starts[G][NW][32];
};

// Named barriers: one of each group, two between the groups' joining warps.
template <int THREADS>
__device__ __forceinline__ void bar_sync(int id) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
template <int THREADS>
__device__ __forceinline__ void bar_arrive(int id) { asm volatile("barrier.cta.arrive %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
constexpr int kGroupBarrier = 1, kCarryBarrier = 3;

// Waits that run out (they cannot, short of a fault: the blocks of a cluster run together) are
// counted here; dgc_gated_scan_check reports them.  Their group takes no further part in the
// exchange (a second arrival in the barrier's phase is not allowed), and stays until every block
// is through: see join_end.
__device__ int g_scan_waits_out;

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

template <int VEC, int NW, int G, int CL>
__device__ __forceinline__ void join_begin(Join<VEC, NW, G, CL>& sm, int ncl) {
  if constexpr (CL > 1) {
    if (ncl == 1) return;
    if (threadIdx.x < G) sm.gone[threadIdx.x] = 0;
    if (threadIdx.x < kBlockSlots)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&sm.arrived[threadIdx.x])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    cg::this_cluster().sync();   // every block runs, its barriers are there
  }
}

__device__ __forceinline__ uint32_t clock_ns() {   // modulo 2^32: 4.3 seconds
  uint32_t t;
  asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
  return t;
}

__device__ __forceinline__ bool wait_arrived(uint32_t barrier, uint32_t phase) {
  uint32_t last = 0, waited = 0;
  while (waited <= kWaitNs) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(barrier), "r"(phase) : "memory");
    if (done) return true;
    const uint32_t now = clock_ns();
    if (last) waited += min(now - last, kPauseNs);
    last = now;
  }
  atomicAdd(&g_scan_waits_out, 1);
  return false;
}

// A group of warps whose wait ran out stays until every other thread of the cluster has come here
// or ended (all waits are bounded, so all do): its block's shared memory may still be stored to.
template <int VEC, int NW, int G, int CL>
__device__ __forceinline__ void join_end(const Join<VEC, NW, G, CL>& sm, int ncl, int group) {
  if constexpr (CL > 1) {
    if (ncl > 1 && sm.gone[group]) asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
  }
}

// Joins the runs of a round in order: takes this warp's map (P, S), returns the state its run
// starts from.  The group's first warp does the work for the block; with one group it keeps
// `carry`, the state before the round, itself, with two it has it from the other group's first
// warp, which joined the round before.  A block's map reaches the others by asynchronous stores
// that complete on their barriers, not through the cluster's barrier: that one would wait for
// every store of results under way.
template <int VEC, int NW, int G, int CL>
__device__ __forceinline__ Val<VEC> join_runs(Join<VEC, NW, G, CL>& sm, int round, bool last, int ncl, int rank, int group,
                                              int warp, int lane, Val<VEC> P, const Val<VEC>& S,
                                              Val<VEC>& carry) {
  P = held(P);
  sm.runs[group][warp][lane] = {P, S};
  bar_sync<NW * 32>(kGroupBarrier + group);
  if (warp == 0) {
    if constexpr (CL > 1) {
      const int slot = round % kBlockSlots;
      if (ncl > 1 && !sm.gone[group]) {
        Val<VEC> tp = P, ts = S;
#pragma unroll
        for (int w = 1; w < NW; ++w) {
          const Map<VEC> m = sm.runs[group][w][lane];
          tp = mul_(m.p, tp);
          ts = fma_(m.p, ts, m.s);
        }
        tp = held(tp);
        const uint32_t to = shared_address(&sm.blocks[slot][rank][lane]), bar = shared_address(&sm.arrived[slot]);
        if (lane == 0)
          asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(ncl * 32 * 2 * VEC * 4) : "memory");
#pragma unroll
        for (int r = 0; r < CL; ++r) {
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
        if (!wait_arrived(bar, (uint32_t)(round / kBlockSlots) & 1u)) sm.gone[group] = 1;
        __syncwarp();
      }
      if (round > 0) {
        bar_sync<64>(kCarryBarrier + (round & 1));
        carry = sm.carry[round & 1][lane];
      }
    }
    Val<VEC> cur = carry;
    const bool several = CL > 1 && ncl > 1;
    if constexpr (CL > 1) {
      if (several) {
#pragma unroll
        for (int r0 = 0; r0 < CL; r0 += 4) {   // (four loads under way at a time)
          if (r0 < ncl) {
            Map<VEC> m[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (r0 + r < ncl) m[r] = sm.blocks[round % kBlockSlots][r0 + r][lane];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if (r0 + r == rank) cur = carry;
              if (r0 + r < ncl) carry = fma_(m[r].p, carry, m[r].s);
            }
          }
        }
        if (!last) {
          sm.carry[(round + 1) & 1][lane] = carry;
          bar_arrive<64>(kCarryBarrier + ((round + 1) & 1));
        }
      }
    }
    constexpr int Q = 4;
#pragma unroll
    for (int w0 = 0; w0 < NW; w0 += Q) {
      Map<VEC> m[Q];
#pragma unroll
      for (int w = 0; w < Q; ++w) m[w] = sm.runs[group][w0 + w][lane];
#pragma unroll
      for (int w = 0; w < Q; ++w) {
        sm.starts[group][w0 + w][lane] = cur;
        cur = fma_(m[w].p, cur, m[w].s);
      }
    }
    if (!several) {
      carry = cur;
      if constexpr (CL > 1) {
        if (!last) {
          sm.carry[(round + 1) & 1][lane] = carry;
          bar_arrive<64>(kCarryBarrier + ((round + 1) & 1));
        }
      }
    }
  }
  bar_sync<NW * 32>(kGroupBarrier + group);
  return sm.starts[group][warp][lane];
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
template <class T, int L, int NW, int G>
struct Place {
  static constexpr int VEC = 4 / sizeof(T);
  int lane, warp, group, ncl, rank, s, c0, c, first, len, mine0, step, width;
  bool on0, on1;
  int64_t at0, dir;
  __device__ __forceinline__ explicit Place(const ScanArgs& a) {
    lane = threadIdx.x & 31;
    warp = (threadIdx.x >> 5) % NW;
    group = (threadIdx.x >> 5) / NW;
    rank = G > 1 && a.cluster > 1 ? (int)(blockIdx.x % a.cluster) : 0;
    const int unit = G > 1 ? blockIdx.x / a.cluster : blockIdx.x;
    s = a.longest_first ? by_length(a, unit / a.ctiles) : unit / a.ctiles;
    c0 = (unit % a.ctiles) * 32 * VEC;
    c = c0 + lane * VEC;
    on0 = c < a.channels;
    on1 = c + 1 < a.channels;
    width = min(32 * VEC, a.channels - c0) * (int)sizeof(T);
    sequence_range(a, s, first, len);
    at0 = a.reverse ? (int64_t)first + len - 1 : first;   // the scan's first token
    dir = a.reverse ? -1 : 1;
    // a short sequence is left to the cluster's first blocks
    constexpr int share = NW * L * G;
    ncl = G > 1 ? min(a.cluster, max(1, (len - 1) / share + 1)) : 1;
    mine0 = ((group * ncl + rank) * NW + warp) * L;
    step = ncl * NW * L * G;   // from one of a group's rounds to its next
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

template <class T, Lie LIE, int L, int NW, int G, int BLOCKS, int CL>
__global__ void __launch_bounds__(NW * G * 32, BLOCKS) k_scan_forward(const ScanArgs a) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), kPart = L * kPitch<LIE>;
  // (on a 128-byte boundary: a row's part that lies across one is read in two steps, 15 % slower)
  extern __shared__ __align__(1024) char buffer[];   // [warp][stage][z, x][L rows]
  __shared__ Join<VEC, NW, G, CL> sm;
  const Place<T, L, NW, G> at(a);
  if (at.rank >= at.ncl) return;
  const int len = at.len;
  const int64_t row0 = at.at0 + at.dir * at.mine0;
  const char* z = first_copy<T, LIE>(a.z, row0, at.c0, a.z.stride, at.lane);
  const char* x = first_copy<T, LIE>(a.x, row0, at.c0, a.x.stride, at.lane);
  // (low halves of addresses: where in their granules the rows of the round in hand start)
  uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(z), x0 = (uint32_t)reinterpret_cast<uintptr_t>(x);
  char* const mine = buffer + (at.group * NW + at.warp) * (kStages * 2 * kPart);
  int ahead = len - at.mine0;   // steps from the next fetch's first on (may be negative)
  auto fetch = [&](int stage) {
    copy_rows<T, LIE, L>(mine + stage * 2 * kPart, z, a.z, a.z.stride, a.z.stride * at.step, 0, min(ahead, L), at.width, at.lane);
    copy_rows<T, LIE, L>(mine + stage * 2 * kPart + kPart, x, a.x, a.x.stride, a.x.stride * at.step, 0, min(ahead, L), at.width, at.lane);
    end_copies();
    ahead = max(ahead - at.step, 0);
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) fetch(i);
  Val<VEC> carry = at.get(a.h0, a.channels);
  if (len == 0) {   // (the same for all blocks of the cluster)
    if (a.h_last && at.rank == 0 && threadIdx.x < 32) at.put(a.h_last, a.channels, carry);
    return;
  }
  join_begin(sm, at.ncl);

  char* out = row_at<T>(a.h, row0, at.c);
  int stage = 0;
  const int rounds = (len - 1) / (at.step / G) + 1;   // of the block
  int left = len - at.mine0;   // steps from this warp's first of the round on
  for (int round = at.group; round < rounds; round += G, left -= at.step) {
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
    z0 += (uint32_t)a.z.stride * (uint32_t)at.step;
    x0 += (uint32_t)a.x.stride * (uint32_t)at.step;
    Val<VEC> cur = join_runs(sm, round, round + 1 == rounds, at.ncl, at.rank, at.group, at.warp, at.lane, P, S, carry);
    auto write = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < L; ++i, out += a.h.stride) {
        cur = fma_(f[i], cur, b[i]);
        if (decltype(whole)::value || i < left) put_word<T, LIE>(out, cur, at.on0, at.on1);
      }
    };
    if (full) write(std::true_type{});
    else write(std::false_type{});
    out += a.h.stride * (at.step - L);
    // (steps after the last have f = 1, b = 0: they pass the state on unchanged)
    if (a.h_last && left > 0 && left <= L) at.put(a.h_last, a.channels, cur);
  }
  wait_copies<0>();
  join_end(sm, at.ncl, at.group);
}

// Backward, walked from the sequence's end: position u = len-1-t.  A thread's run of L steps
// needs h_{t-1} at each of them; it reads the stored h once, before the run's first step, and
// recomputes the others in 32 bits from z and x, which it has to read anyway: 5 words moved a
// step instead of 6, and the states inside a run carry no rounding of the output type.  The one
// before it does: of 65536 x 2048 bf16 dgate is 1.73e-3 from its 64-bit values in the 2-norm, where
// states of 32 bits throughout, rounded at the end as here, would give 1.66e-3.
template <class T, Lie LIE, int L, int NW, int G, int BLOCKS, int CL>
__global__ void __launch_bounds__(NW * G * 32, BLOCKS) k_scan_backward(const ScanArgs a) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), kPart = L * kPitch<LIE>;
  // (on a 128-byte boundary: a row's part that lies across one is read in two steps, 15 % slower)
  extern __shared__ __align__(1024) char buffer[];   // [warp][stage][z, x, dh][L rows]
  __shared__ Join<VEC, NW, G, CL> sm;
  const Place<T, L, NW, G> at(a);
  if (at.rank >= at.ncl) return;
  const int len = at.len;
  // a stage holds the steps t_lo .. t_lo + L - 1 in ascending order; the rounds descend
  const int64_t row0 = at.at0 + at.dir * (int64_t)(len - L - at.mine0);
  const char* z = first_copy<T, LIE>(a.z, row0, at.c0, a.z.stride, at.lane);
  const char* x = first_copy<T, LIE>(a.x, row0, at.c0, a.x.stride, at.lane);
  const char* d = first_copy<T, LIE>(a.dh, row0, at.c0, a.dh.stride, at.lane);
  uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(z), x0 = (uint32_t)reinterpret_cast<uintptr_t>(x),
           d0 = (uint32_t)reinterpret_cast<uintptr_t>(d);
  char* const mine = buffer + (at.group * NW + at.warp) * (kStages * 3 * kPart);
  int ahead = len - at.mine0;   // steps of the next fetch and before it (may be negative)
  auto fetch = [&](int stage) {
    char* to = mine + stage * 3 * kPart;
    const int lo = ahead > 0 ? max(L - ahead, 0) : L;
    copy_rows<T, LIE, L>(to, z, a.z, a.z.stride, -a.z.stride * at.step, lo, L, at.width, at.lane);
    copy_rows<T, LIE, L>(to + kPart, x, a.x, a.x.stride, -a.x.stride * at.step, lo, L, at.width, at.lane);
    copy_rows<T, LIE, L>(to + 2 * kPart, d, a.dh, a.dh.stride, -a.dh.stride * at.step, lo, L, at.width, at.lane);
    end_copies();
    ahead = max(ahead - at.step, 0);
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) fetch(i);
  Val<VEC> carry = at.get(a.dh_last, a.channels);
  const Val<VEC> start = at.get(a.h0, a.channels);
  if (len == 0) {
    if (a.dh0 && at.rank == 0 && threadIdx.x < 32) at.put(a.dh0, a.channels, carry);
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
  int stage = 0;
  const int rounds = (len - 1) / (at.step / G) + 1;   // of the block
  for (int round = at.group; round < rounds; round += G, left -= at.step) {
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
    Val<VEC> cur = join_runs(sm, round, round + 1 == rounds, at.ncl, at.rank, at.group, at.warp, at.lane, P, S, carry);
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
    gz -= a.dz.stride * (at.step - L);
    gx -= a.dx.stride * (at.step - L);
    if (a.dh0 && left > 0 && left <= L) at.put(a.dh0, a.channels, cur);
    __syncwarp();   // the stage has been read by all lanes
    fetch(stage);
    stage ^= 1;
    z0 -= (uint32_t)a.z.stride * (uint32_t)at.step;
    x0 -= (uint32_t)a.x.stride * (uint32_t)at.step;
    d0 -= (uint32_t)a.dh.stride * (uint32_t)at.step;
  }
  wait_copies<0>();
  join_end(sm, at.ncl, at.group);
}

// ------------------------------------------------------------------ few and narrow sequences
// A few long sequences of few channels leave most SMs idle above, and a cluster's rounds are a
// chain.  With a workspace they are cut into runs of kRun steps that any warp can take: one kernel
// reduces every run to its map, one joins the maps of a sequence and leaves every run's start, one
// walks the runs again from there and writes.  The rows are read twice, the second time mostly out
// of L2; which calls take this way, and what it measured, stands at wide_bytes.
constexpr int kRun = 64, kWideWarps = 4, kJoinWarps = 16;

// Run c of sequence s has the slot first / kRun + s + c: different ones for all runs, below
// tokens / kRun + seqs.
struct WideArgs {
  ScanArgs a;
  float2* maps;      // [slots][channels]: P and S; after the join, P is the start
};

template <class T>
struct WidePlace {   // a warp's run and channels
  static constexpr int VEC = 4 / sizeof(T);
  int lane, s, c0, c, first, len, at, width;   // at: the run's first step
  bool on0, on1, any;
  int64_t slot, at0, dir;
  __device__ __forceinline__ explicit WidePlace(const ScanArgs& a) {
    lane = threadIdx.x & 31;
    slot = (int64_t)blockIdx.x * kWideWarps + (threadIdx.x >> 5);
    c0 = blockIdx.y * 32 * VEC;
    c = c0 + lane * VEC;
    on0 = c < a.channels;
    on1 = c + 1 < a.channels;
    width = min(32 * VEC, a.channels - c0) * (int)sizeof(T);
    any = false;
    for (int q0 = 0; q0 < a.seqs && !any; q0 += 32) {   // whose run is it: 32 sequences at a time
      const int q = q0 + lane;
      int f = 0, l = 0;
      if (q < a.seqs) sequence_range(a, q, f, l);
      const int64_t run = slot - (f / kRun + q);
      const uint32_t hit = __ballot_sync(0xFFFFFFFFu, q < a.seqs && run >= 0 && run * kRun < l);
      if (hit) {
        const int who = __ffs(hit) - 1;
        any = true;
        s = q0 + who;
        first = __shfl_sync(0xFFFFFFFFu, f, who);
        len = __shfl_sync(0xFFFFFFFFu, l, who);
        at = (int)(__shfl_sync(0xFFFFFFFFu, (int)run, who) * kRun);
      }
    }
    if (any) {
      at0 = a.reverse ? (int64_t)first + len - 1 : first;
      dir = a.reverse ? -1 : 1;
    }
  }
};

// Maps of the runs: forward of z and x, backward of z and dh (walked from the run's end).
template <class T, Lie LIE, bool BACK>
__global__ void __launch_bounds__(kWideWarps * 32) k_wide_reduce(const WideArgs w) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), L = 16, kPart = L * kPitch<LIE>;
  __shared__ __align__(128) char buffer[kWideWarps][2][2][kPart];
  const ScanArgs& a = w.a;
  const WidePlace<T> at(a);
  if (!at.any) return;   // (a warp on its own: nothing below waits for another)
  const Matrix& second = BACK ? a.dh : a.x;
  char (*mine)[2][kPart] = buffer[threadIdx.x >> 5];
  const int n = min(at.len - at.at, kRun);             // steps of the run
  const int stages = (n + L - 1) / L;
  const auto stage_of = [&](int i) { return BACK ? stages - 1 - i : i; };
  const auto fetch = [&](int i) {
    if (i < stages) {
      const int64_t row = at.at0 + at.dir * (int64_t)(at.at + stage_of(i) * L);
      const int hi = min(n - stage_of(i) * L, L);
      const char* p = first_copy<T, LIE>(a.z, row, at.c0, a.z.stride, at.lane);
      copy_rows<T, LIE, L>(mine[i & 1][0], p, a.z, a.z.stride, 0, 0, hi, at.width, at.lane);
      p = first_copy<T, LIE>(second, row, at.c0, second.stride, at.lane);
      copy_rows<T, LIE, L>(mine[i & 1][1], p, second, second.stride, 0, 0, hi, at.width, at.lane);
    }
    end_copies();
  };
  fetch(0);
  fetch(1);
  Val<VEC> P = fill<VEC>(1.0f), S = fill<VEC>(0.0f);
  for (int i = 0; i < stages; ++i) {
    wait_copies<1>();
    const int t0 = stage_of(i) * L;
    const int64_t row = at.at0 + at.dir * (int64_t)(at.at + t0);
    const uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(a.z, row, at.c0));
    const uint32_t y0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(second, row, at.c0));
#pragma unroll
    for (int k = 0; k < L; ++k) {
      const int j = BACK ? L - 1 - k : k;
      Val<VEC> f, omf;
      gate(row_word<T, LIE>(mine[i & 1][0], z0, (uint32_t)a.z.stride, j, at.lane), f, omf);
      const Val<VEC> y = row_word<T, LIE>(mine[i & 1][1], y0, (uint32_t)second.stride, j, at.lane);
      if (t0 + j < n) {
        P = mul_(P, f);
        S = BACK ? mul_(f, add_(y, S)) : fma_(f, S, mul_(omf, y));
      }
    }
    __syncwarp();
    fetch(i + 2);
  }
  wait_copies<0>();
  float2* m = w.maps + at.slot * a.channels + at.c;
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    if (v ? at.on1 : at.on0) m[v] = make_float2(held(P.v[v]), S.v[v]);
}

// The starts of a sequence's runs, in the order of the walk, and the state after the last.
__global__ void __launch_bounds__(kJoinWarps * 32) k_wide_join(const WideArgs w, int back) {
  pdl_enter();
  __shared__ float2 parts[kJoinWarps][32];
  const ScanArgs& a = w.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.y, c = blockIdx.x * 32 + lane;
  const bool on = c < a.channels;
  int first, len;
  sequence_range(a, s, first, len);
  const int runs = (len + kRun - 1) / kRun, share = (runs + kJoinWarps - 1) / kJoinWarps;
  const int lo = min(warp * share, runs), hi = min(lo + share, runs);
  float2* maps = w.maps + (int64_t)(first / kRun + s) * a.channels + c;
  const auto map = [&](int i) -> float2& { return maps[(int64_t)(back ? runs - 1 - i : i) * a.channels]; };
  float2 t = make_float2(1.0f, 0.0f);
  if (on) {
#pragma unroll 8
    for (int i = lo; i < hi; ++i) {
      const float2 m = map(i);
      t = make_float2(m.x * t.x, fmaf(m.x, t.y, m.y));
    }
  }
  parts[warp][lane] = make_float2(held(t.x), t.y);
  __syncthreads();
  if (!on) return;
  const float* from = back ? a.dh_last : a.h0;
  float cur = from ? from[(int64_t)s * a.channels + c] : 0.0f;
  for (int q = 0; q < warp; ++q) cur = fmaf(parts[q][lane].x, cur, parts[q][lane].y);
  for (int i0 = lo; i0 < hi; i0 += 8) {   // eight loads before the stores that they could meet
    float2 m[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = map(min(i0 + k, hi - 1));
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k < hi) {
        map(i0 + k).x = cur;
        cur = fmaf(m[k].x, cur, m[k].y);
      }
  }
  float* to = back ? a.dh0 : a.h_last;
  if (to && warp == kJoinWarps - 1) to[(int64_t)s * a.channels + c] = cur;
}

template <class T, Lie LIE>
__global__ void __launch_bounds__(kWideWarps * 32) k_wide_forward(const WideArgs w) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), L = 16, kPart = L * kPitch<LIE>;
  __shared__ __align__(128) char buffer[kWideWarps][2][2][kPart];
  const ScanArgs& a = w.a;
  const WidePlace<T> at(a);
  if (!at.any) return;
  char (*mine)[2][kPart] = buffer[threadIdx.x >> 5];
  const int n = min(at.len - at.at, kRun), stages = (n + L - 1) / L;
  const auto fetch = [&](int i) {
    if (i < stages) {
      const int64_t row = at.at0 + at.dir * (int64_t)(at.at + i * L);
      const int hi = min(n - i * L, L);
      const char* p = first_copy<T, LIE>(a.z, row, at.c0, a.z.stride, at.lane);
      copy_rows<T, LIE, L>(mine[i & 1][0], p, a.z, a.z.stride, 0, 0, hi, at.width, at.lane);
      p = first_copy<T, LIE>(a.x, row, at.c0, a.x.stride, at.lane);
      copy_rows<T, LIE, L>(mine[i & 1][1], p, a.x, a.x.stride, 0, 0, hi, at.width, at.lane);
    }
    end_copies();
  };
  fetch(0);
  fetch(1);
  const float2* m = w.maps + at.slot * a.channels + at.c;
  Val<VEC> cur;
#pragma unroll
  for (int v = 0; v < VEC; ++v) cur.v[v] = (v ? at.on1 : at.on0) ? m[v].x : 0.0f;
  char* out = row_at<T>(a.h, at.at0 + at.dir * (int64_t)at.at, at.c);
  for (int i = 0; i < stages; ++i) {
    wait_copies<1>();
    const int64_t row = at.at0 + at.dir * (int64_t)(at.at + i * L);
    const uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(a.z, row, at.c0));
    const uint32_t x0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(a.x, row, at.c0));
#pragma unroll
    for (int j = 0; j < L; ++j, out += a.h.stride) {
      Val<VEC> f, omf;
      gate(row_word<T, LIE>(mine[i & 1][0], z0, (uint32_t)a.z.stride, j, at.lane), f, omf);
      cur = fma_(f, cur, mul_(omf, row_word<T, LIE>(mine[i & 1][1], x0, (uint32_t)a.x.stride, j, at.lane)));
      if (i * L + j < n) put_word<T, LIE>(out, cur, at.on0, at.on1);
    }
    __syncwarp();
    fetch(i + 2);
  }
  wait_copies<0>();
}

template <class T, Lie LIE>
__global__ void __launch_bounds__(kWideWarps * 32) k_wide_backward(const WideArgs w) {
  pdl_enter();
  constexpr int VEC = 4 / sizeof(T), L = 8, kPart = L * kPitch<LIE>;
  __shared__ __align__(128) char buffer[kWideWarps][2][3][kPart];
  const ScanArgs& a = w.a;
  const WidePlace<T> at(a);
  if (!at.any) return;
  char (*mine)[3][kPart] = buffer[threadIdx.x >> 5];
  const int n = min(at.len - at.at, kRun), stages = (n + L - 1) / L;
  uint32_t before[2] = {0, 0};   // the stored state before the next stage's first step, as it lies
  const auto fetch_state = [&](int i) {
    const int64_t t = at.at + (stages - 1 - i) * L - 1;
    if (i < stages && t >= 0) {
      const T* p = reinterpret_cast<const T*>(row_at<T>(a.h, at.at0 + at.dir * t, at.c));
      if constexpr (LIE == kHalves) {
        if (at.on0) before[0] = load_word<T, 1>(p);
        if (at.on1) before[1] = load_word<T, 1>(p + 1);
      } else {
        if (at.on0) before[0] = load_word<T, VEC>(p);
      }
    }
  };
  const auto fetch = [&](int i) {
    if (i < stages) {
      const int64_t row = at.at0 + at.dir * (int64_t)(at.at + (stages - 1 - i) * L);
      const int hi = min(n - (stages - 1 - i) * L, L);
      const Matrix* from[3] = {&a.z, &a.x, &a.dh};
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const char* p = first_copy<T, LIE>(*from[q], row, at.c0, from[q]->stride, at.lane);
        copy_rows<T, LIE, L>(mine[i & 1][q], p, *from[q], from[q]->stride, 0, 0, hi, at.width, at.lane);
      }
    }
    end_copies();
  };
  fetch(0);
  fetch(1);
  fetch_state(0);
  const float2* m = w.maps + at.slot * a.channels + at.c;
  Val<VEC> cur, start;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    const bool on = v ? at.on1 : at.on0;
    cur.v[v] = on ? m[v].x : 0.0f;
    start.v[v] = on && a.h0 ? a.h0[(int64_t)at.s * a.channels + at.c + v] : 0.0f;
  }
  for (int i = 0; i < stages; ++i) {
    const int t0 = (stages - 1 - i) * L;
    const int64_t row = at.at0 + at.dir * (int64_t)(at.at + t0);
    const uint32_t z0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(a.z, row, at.c0));
    const uint32_t x0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(a.x, row, at.c0));
    const uint32_t d0 = (uint32_t)reinterpret_cast<uintptr_t>(row_at<T>(a.dh, row, at.c0));
    Val<VEC> hp, f[L], omf[L], e[L];
    if constexpr (LIE == kHalves) unpack<T, 2>(before[0] | before[1] << 16, hp.v);
    else unpack<T, VEC>(before[0], hp.v);
    if (at.at + t0 == 0) hp = start;
    fetch_state(i + 1);
    wait_copies<1>();
#pragma unroll
    for (int j = 0; j < L; ++j) {
      gate(row_word<T, LIE>(mine[i & 1][0], z0, (uint32_t)a.z.stride, j, at.lane), f[j], omf[j]);
      const Val<VEC> x_t = row_word<T, LIE>(mine[i & 1][1], x0, (uint32_t)a.x.stride, j, at.lane);
      e[j] = sub_(hp, x_t);
      hp = fma_(f[j], hp, mul_(omf[j], x_t));   // (past the run's end: not used)
    }
    char* gz = row_at<T>(a.dz, row + at.dir * (L - 1), at.c);
    char* gx = row_at<T>(a.dx, row + at.dir * (L - 1), at.c);
#pragma unroll
    for (int j = L - 1; j >= 0; --j, gz -= a.dz.stride, gx -= a.dx.stride) {
      if (t0 + j < n) {
        const Val<VEC> gt = add_(row_word<T, LIE>(mine[i & 1][2], d0, (uint32_t)a.dh.stride, j, at.lane), cur);
        cur = mul_(f[j], gt);
        put_word<T, LIE>(gx, mul_(omf[j], gt), at.on0, at.on1);
        put_word<T, LIE>(gz, mul_(mul_(omf[j], cur), e[j]), at.on0, at.on1);
      }
    }
    __syncwarp();
    fetch(i + 2);
  }
  wait_copies<0>();
}

// One token a sequence: the state is read, advanced and written back where it lies.  A thread
// takes N neighbouring channels (4, in words of 16 bytes of state, where everything is aligned
// for that), a block's rows are given by the grid's second dimension: no divisions.
template <class T, int N>
__global__ void __launch_bounds__(256)
k_scan_step(const T* z, int64_t ld_z, const T* x, int64_t ld_x, float* state, const int32_t* slots,
            int32_t num_slots, T* out, int64_t ld_out, int32_t rows, int32_t channels) {
  pdl_enter();
  const int c = (blockIdx.x * 256 + threadIdx.x) * N;
  if (c >= channels) return;
  for (unsigned r = blockIdx.y; r < (unsigned)rows; r += gridDim.y) {
    const int slot = slots ? __ldg(slots + r) : (int)r;
    const bool live = slot >= 0 && slot < num_slots;
    float* st = state + (int64_t)(live ? slot : 0) * channels + c;
    struct alignas(sizeof(T) * N) Pack { T v[N]; };
    struct alignas(4 * N) State { float v[N]; };
    const Pack zw = *reinterpret_cast<const Pack*>(z + r * ld_z + c), xw = *reinterpret_cast<const Pack*>(x + r * ld_x + c);
    State h{};
    if (live) h = *reinterpret_cast<const State*>(st);
    Pack o;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      Val<1> f, omf;
      gate(Val<1>{{to_float<T>(zw.v[i])}}, f, omf);
      h.v[i] = live ? fmaf(f.v[0], h.v[i], omf.v[0] * to_float<T>(xw.v[i])) : 0.0f;
      o.v[i] = from_float<T>(h.v[i]);
    }
    if (live) *reinterpret_cast<State*>(st) = h;
    *reinterpret_cast<Pack*>(out + r * ld_out + c) = o;
  }
}

// The last tile of channels ends below 2^31 (a block of k_scan_step takes 1024).
constexpr int32_t kMaxChannels = INT32_MAX - 1024;
inline bool bad_channels(int32_t channels) { return channels < 1 || channels > kMaxChannels; }

constexpr int kFwdL = 16, kBwdL = 8, kSms = 148;
constexpr int kWideUnits = 16, kWideShort = 2048, kWideLong = 8192, kWideWork = 32768;

template <class T>
void lay_out(ScanArgs& a) {
  for (Matrix* m : {&a.z, &a.x, &a.h, &a.dh, &a.dz, &a.dx}) {
    m->end = m->begin + ((int64_t)(a.tokens - 1) * m->ld + a.channels) * (int64_t)sizeof(T);
    m->stride = (a.reverse ? -m->ld : m->ld) * (int64_t)sizeof(T);
  }
}

// Bytes of workspace with which a call goes by runs; 0 where it would not.  Its three launches take
// 9 us forward and 13 backward at the least, whatever they work on; a cluster a sequence takes
// (forward / backward, runs against clusters, bf16 unless stated, in a graph)
//   60000 steps x  100 f16   36 / 46 against 68 / 112 us      8192 x  256    9.3 / 13.8 against 9.4 / 13.9
//   30000 x 1024             68 / 91 against 81 / 131         4096 x  256    9.8 / 13.9 against 6.7 /  9.3
//   16384 x   64 f16        9.8 / 14 against 14 /  23         2048 x 1024    9.3 / 13.4 against 10.8 / 15.0
int64_t wide_bytes(int64_t tokens, int32_t seqs, int32_t channels, size_t es) {
  const int32_t words = 128 / (int32_t)es;
  const int64_t units = (int64_t)((channels + words - 1) / words) * seqs;
  const int64_t len = tokens / seqs;
  if (units > kWideUnits || len < kWideShort || (len < kWideLong && len * units < kWideWork)) return 0;
  return (tokens / kRun + seqs) * channels * (int64_t)sizeof(float2);
}

template <class T, Lie LIE>
int32_t enqueue_wide(ScanArgs a, float2* maps, bool backward, cudaStream_t s) {
  lay_out<T>(a);
  const WideArgs w{a, maps};
  constexpr int words = 128 / (int)sizeof(T);
  const int64_t slots = (int64_t)a.tokens / kRun + a.seqs;
  const dim3 grid((unsigned)((slots + kWideWarps - 1) / kWideWarps), (a.channels + words - 1) / words);
  const dim3 threads(kWideWarps * 32), join((a.channels + 31) / 32, a.seqs);
  if (backward) launch(k_wide_reduce<T, LIE, true>, grid, threads, 0, s, w);
  else launch(k_wide_reduce<T, LIE, false>, grid, threads, 0, s, w);
  int32_t rc = check_launch();
  if (rc != DGC_OK) return rc;
  launch(k_wide_join, join, dim3(kJoinWarps * 32), 0, s, w, backward ? 1 : 0);
  if ((rc = check_launch()) != DGC_OK) return rc;
  if (backward) launch(k_wide_backward<T, LIE>, grid, threads, 0, s, w);
  else launch(k_wide_forward<T, LIE>, grid, threads, 0, s, w);
  return check_launch();
}

template <class T, Lie LIE, int NW, int G, int CL>
int32_t enqueue(ScanArgs a, bool backward, cudaStream_t s) {
  constexpr int VEC = 4 / sizeof(T), BLOCKS = 16 / (NW * G);   // 16 warps of 128 registers an SM
  const int L = backward ? kBwdL : kFwdL;
  a.ctiles = (a.channels + 32 * VEC - 1) / (32 * VEC);
  const int64_t units = (int64_t)a.ctiles * a.seqs;
  // As many blocks of a cluster as there are SMs for, and steps: 4 blocks a sequence instead of 1
  // take 65536 x 2048 bf16 from 515 to 164 us; where the SMs have enough to do without, the
  // exchange costs (40 -> 56 us for 16 x 1024 x 1001).
  a.cluster = 1;
  if (CL > 1)
    while (a.cluster < CL && units * (a.cluster + 1) <= kSms &&
           (int64_t)a.cluster * (L * NW * G) < a.tokens / a.seqs)
      ++a.cluster;
  a.longest_first = a.seq_start && a.seqs > 1 && a.seqs <= kSorted && units > kSms;
  int64_t grid = units * a.cluster;
  if (grid > INT32_MAX) return DGC_EINVAL;
  lay_out<T>(a);
  const size_t smem = G * NW * kStages * kPitch<LIE> * (backward ? 3 * kBwdL : 2 * kFwdL);
  auto go = [&](auto kernel) {
    constexpr auto f = decltype(kernel)::value;
    const int32_t rc = allow_shared<f>(smem);
    if (rc != DGC_OK) return rc;
    if constexpr (CL > kPortableCluster) {
      if (!allow_cluster<f>(CL, NW * G * 32, smem)) {
        a.cluster = std::min(a.cluster, kPortableCluster);
        grid = units * a.cluster;
      }
    }
    const dim3 blocks((unsigned)grid), threads(NW * G * 32);
    if (CL > 1 && a.cluster > 1) launch_cluster(f, blocks, threads, smem, s, (unsigned)a.cluster, a);
    else launch(f, blocks, threads, smem, s, a);
    return check_launch();
  };
  using Kernel = void (*)(ScanArgs);
  if (backward) return go(std::integral_constant<Kernel, &k_scan_backward<T, LIE, kBwdL, NW, G, BLOCKS, CL>>{});
  return go(std::integral_constant<Kernel, &k_scan_forward<T, LIE, kFwdL, NW, G, BLOCKS, CL>>{});
}

// Which blocks.  All have 16 warps of 128 registers an SM; they differ in how many of them work at
// one sequence (forward / backward, bf16 unless stated):
//   four blocks of 4 warps   where there are blocks for all slots, or runs end early:
//                            32 x 1024 steps x 1024 channels 36 / 60 us against 36 / 64 with 8 warps,
//                            20 x 35 x 1500 f32 4.6 / 7.3 against 8.5 / 9.4
//   two blocks of 8 warps    in between: 16 x 512 x 1024 12 / 19 us against 13 / 22 with 4 warps and
//                            16 / 23 with 16
//   one block of 2 x 8 warps puts a whole SM behind a sequence, where they are long and few, or uneven
//                            (the longest then decides): 20 of 500 on average x 1024 19 / 27 us against
//                            22 / 43 with 4 warps; clusters are for these
// More blocks of a cluster than the portable eight where next to nothing else is there to do
// (69 against 131 us for one sequence of 60000 x 100 f16 without a workspace); beyond four clusters of sixteen not all
// find room at once (8 of them: 19 against 14 us for 8192 x 512).
template <class T, Lie LIE>
int32_t enqueue(const ScanArgs& a, float2* maps, bool backward, cudaStream_t s) {
  if (maps) return enqueue_wide<T, LIE>(a, maps, backward, s);
  const int32_t len = a.tokens / a.seqs, words = 32 * 4 / (int)sizeof(T);
  const int64_t units = (int64_t)((a.channels + words - 1) / words) * a.seqs;
  const bool uneven = a.seq_start != nullptr;
  if (len <= 64 || (units >= 500 && len <= (uneven ? 200 : 1024)))
    return enqueue<T, LIE, 4, 1, 1>(a, backward, s);
  if (len < (uneven ? 400 : 640) && (len <= 128 || units >= kSms))
    return enqueue<T, LIE, 8, 1, 1>(a, backward, s);
  if (units <= 4 && len > 1024) return enqueue<T, LIE, 8, 2, kMaxCluster>(a, backward, s);
  return enqueue<T, LIE, 8, 2, kPortableCluster>(a, backward, s);
}

int32_t dispatch(const ScanArgs& a, float2* maps, int32_t dtype, bool backward, Lie lie, cudaStream_t s) {
  if (dtype == DGC_F32)
    return lie == kAligned ? enqueue<float, kAligned>(a, maps, backward, s) : enqueue<float, kWords>(a, maps, backward, s);
  if (dtype == DGC_BF16)
    return lie == kAligned ? enqueue<__nv_bfloat16, kAligned>(a, maps, backward, s)
           : lie == kWords ? enqueue<__nv_bfloat16, kWords>(a, maps, backward, s)
                           : enqueue<__nv_bfloat16, kHalves>(a, maps, backward, s);
  return lie == kAligned ? enqueue<__half, kAligned>(a, maps, backward, s)
         : lie == kWords ? enqueue<__half, kWords>(a, maps, backward, s)
                         : enqueue<__half, kHalves>(a, maps, backward, s);
}

Matrix matrix(const dgc_matrix& m) { return Matrix{static_cast<char*>(m.data), nullptr, m.ld, 0}; }

// The worst lie of the call's matrices.
Lie lie_of(std::initializer_list<Matrix> ms, int32_t channels, size_t es) {
  size_t bits = channels * es;
  for (const Matrix& m : ms) bits |= reinterpret_cast<uintptr_t>(m.begin) | (size_t)m.ld * es;
  return bits % 16 == 0 ? kAligned : bits % 4 == 0 ? kWords : kHalves;
}

int32_t scan(const dgc_scan* d, bool backward, void* stream) {
  if (!d || bad_dtype(d->dtype) || d->tokens < 0 || d->tokens > INT32_MAX || d->num_seqs < 1 || bad_channels(d->channels) ||
      (!d->seq_start && d->tokens % d->num_seqs != 0))
    return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  const auto bad = [&](const dgc_matrix& m) { return bad_matrix(m, d->tokens, d->channels, es); };
  if (bad(d->gate) || bad(d->x) || bad(d->h) || misaligned(d->h0, 4) || misaligned(d->seq_start, 4) ||
      misaligned(d->workspace, 8) || d->workspace_bytes < 0)
    return DGC_EINVAL;
  if (backward ? bad(d->dh) || bad(d->dgate) || bad(d->dx) || misaligned(d->dh_last, 4) || misaligned(d->dh0, 4)
               : misaligned(d->h_last, 4))
    return DGC_EINVAL;
  if (d->tokens == 0 && !(backward ? d->dh0 : d->h_last)) return DGC_OK;
  ScanArgs a{};
  a.z = matrix(d->gate); a.x = matrix(d->x); a.h = matrix(d->h);
  a.h0 = d->h0; a.seq_start = d->seq_start;
  a.tokens = (int32_t)d->tokens; a.seqs = d->num_seqs; a.seq_len = (int32_t)(d->tokens / d->num_seqs);
  a.channels = d->channels; a.reverse = d->reverse != 0;
  const int64_t wide = d->workspace ? wide_bytes(d->tokens, d->num_seqs, d->channels, es) : 0;
  if (wide && d->workspace_bytes < wide) return DGC_ECAPACITY;
  float2* const maps = wide ? static_cast<float2*>(d->workspace) : nullptr;
  if (!backward) {
    a.h_last = d->h_last;
    return dispatch(a, maps, d->dtype, false, lie_of({a.z, a.x, a.h}, a.channels, es), as_stream(stream));
  }
  a.dh = matrix(d->dh); a.dz = matrix(d->dgate); a.dx = matrix(d->dx);
  a.dh_last = d->dh_last; a.dh0 = d->dh0;
  return dispatch(a, maps, d->dtype, true, lie_of({a.z, a.x, a.h, a.dh, a.dz, a.dx}, a.channels, es), as_stream(stream));
}

}  // namespace

extern "C" {

int32_t dgc_gated_scan_forward(const dgc_scan* d, void* stream) { return scan(d, false, stream); }
int32_t dgc_gated_scan_backward(const dgc_scan* d, void* stream) { return scan(d, true, stream); }

int64_t dgc_gated_scan_workspace_bytes(const dgc_scan* d) {
  if (!d || bad_dtype(d->dtype) || d->tokens < 0 || d->tokens > INT32_MAX || d->num_seqs < 1 || bad_channels(d->channels))
    return DGC_EINVAL;
  return wide_bytes(d->tokens, d->num_seqs, d->channels, element_size(d->dtype));
}

int32_t dgc_gated_scan_step(const dgc_scan_one* d, void* stream) {
  if (!d || bad_dtype(d->dtype) || d->rows < 0 || bad_channels(d->channels) || d->num_slots < 0) return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  if (bad_matrix(d->gate, d->rows, d->channels, es) || bad_matrix(d->x, d->rows, d->channels, es) ||
      bad_matrix(d->out, d->rows, d->channels, es) || misaligned(d->slots, 4))
    return DGC_EINVAL;
  if (d->rows == 0) return DGC_OK;
  if (!d->state || misaligned(d->state, 4) || (!d->slots && d->num_slots < d->rows)) return DGC_EINVAL;
  size_t bits = d->channels * es;
  for (const dgc_matrix& m : {d->gate, d->x, d->out}) bits |= reinterpret_cast<uintptr_t>(m.data) | (size_t)m.ld * es;
  const bool four = bits % (4 * es) == 0 && !misaligned(d->state, 16);
  auto go = [&](auto tag, auto n) {
    using T = decltype(tag);
    constexpr int N = decltype(n)::value;
    const dim3 grid((d->channels + 256 * N - 1) / (256 * N), std::min(d->rows, 65535));
    launch(k_scan_step<T, N>, grid, 256, 0, as_stream(stream), static_cast<const T*>(d->gate.data), d->gate.ld,
           static_cast<const T*>(d->x.data), d->x.ld, d->state, d->slots, d->num_slots, static_cast<T*>(d->out.data),
           d->out.ld, d->rows, d->channels);
  };
  using one = std::integral_constant<int, 1>;
  using all = std::integral_constant<int, 4>;
  if (d->dtype == DGC_F32) four ? go(float{}, all{}) : go(float{}, one{});
  else if (d->dtype == DGC_BF16) four ? go(__nv_bfloat16{}, all{}) : go(__nv_bfloat16{}, one{});
  else four ? go(__half{}, all{}) : go(__half{}, one{});
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
