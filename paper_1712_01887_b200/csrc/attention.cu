// Linear attention with a decay for each head (sm_100a): kernels and C ABI.  The mathematics stands in
// attention.cuh.

#include <algorithm>
#include <cmath>

#include "attention_tensor.cuh"

using namespace dgc;

namespace {

// ------------------------------------------------------------------ the walk in 32-bit arithmetic
// For 32-bit tensors and rows that tensor copies cannot fetch.  A block walks one item (a sequence, or a part of it) of one head and 64
// of the rows' elements, in chunks of 32 tokens.  A thread holds 8 x 4 elements of the state in registers, and forms 2 x 2
// of P and 2 x 4 of the rows; factors come from shared memory four at a time.  All loads of a chunk are under way at
// once (20 x 35 x 12 x 125 f32, forward and backward: 209 us, 379 with loads one after the other and single rows).
constexpr int kC = 32, kDy = 64, kDyPitch = kDy + 4, kThreads = 256, kPPitch = kC + 4;

__host__ __device__ inline int pitch_of(int du) { return (du + 3) / 4 * 4 + 4; }
inline size_t walk_shared(int du) {
  return sizeof(float) * (2 * kC * pitch_of(du) + kC * kDyPitch + kC * kPPitch + DGC_MAX_HEAD_DIM * kDyPitch + kC + 1);
}

// 32 rows, a warp each fourth part of eight; WIDE: 128 columns, else 64.
template <class T, bool WIDE>
struct Fetched {
  static constexpr int N = WIDE ? 4 : 2;
  T v[4][N];
  __device__ __forceinline__ void load(const Heads& from, int h, int token, int n, int d0, int d) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const T* p = static_cast<const T*>(from.p) + (int64_t)token * from.ld + (int64_t)h * from.head + d0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const int row = warp + 8 * i, col = lane + 32 * c;
        v[i][c] = row < n && col < d ? p[(int64_t)row * from.ld + col] : from_float<T>(0.0f);
      }
  }
  __device__ __forceinline__ void store(float* to, int pitch, int width) const {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (lane + 32 * c < width) to[(warp + 8 * i) * pitch + lane + 32 * c] = to_float<T>(v[i][c]);
  }
};

__device__ __forceinline__ void add4(float (&to)[4], float by, const float4& v) {
  to[0] = fmaf(by, v.x, to[0]);
  to[1] = fmaf(by, v.y, to[1]);
  to[2] = fmaf(by, v.z, to[2]);
  to[3] = fmaf(by, v.w, to[3]);
}

// STATES: only the states are wanted, from 0 (a part's own share).
template <class T, bool STATES>
__global__ void __launch_bounds__(kThreads, 2) k_walk(const __grid_constant__ WalkArgs a) {
  pdl_enter();
  extern __shared__ __align__(16) float sm[];
  const Walk& w = a.w[blockIdx.y];
  const int slice = blockIdx.x % a.slices, rest = blockIdx.x / a.slices, h = rest % a.heads, item = rest / a.heads;
  const Item it = item_of(a, item);
  const int du = w.du, y0 = slice * kDy, dy = min(w.dy - y0, kDy);
  if (dy <= 0 || (a.part && it.len == 0)) return;
  const int up = pitch_of(du), du4 = up - 4;
  float* U = sm;
  float* X = U + kC * up;
  float* Y = X + kC * up;
  float* P = Y + kC * kDyPitch;
  float* Z = P + kC * kPPitch;
  float* power = Z + DGC_MAX_HEAD_DIM * kDyPitch;   // g^0 .. g^C
  const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
  const float lg = log_decay(a.decay, h);
  if (tid <= kC) power[tid] = exp2f(tid * lg);
  const int64_t at = ((int64_t)(a.part ? item : it.s) * a.heads + h) * du * w.dy;
  const auto row_of = [&](int i) { return i / 4 * 64 + ty * 4 + i % 4; };   // of the state's, the thread's i-th
  float z[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int r = row_of(i), col = tx * 4 + c;
      z[i][c] = !STATES && w.z_in && r < du && col < dy
                    ? w.z_in[at + (w.turned ? (int64_t)(y0 + col) * du + r : (int64_t)r * w.dy + y0 + col)] : 0.0f;
    }
  const int chunks = (it.len + kC - 1) / kC;
  for (int t = 0; t < chunks; ++t) {
    const int chunk = w.late ? chunks - 1 - t : t, token = it.first + chunk * kC, n = min(kC, it.len - chunk * kC);
    Fetched<T, true> u, x;
    Fetched<T, false> y;
    if (!STATES) u.load(w.u, h, token, n, 0, du);
    x.load(w.x, h, token, n, 0, du);
    y.load(w.y, h, token, n, y0, dy);
    __syncthreads();
    if (!STATES) u.store(U, up, du4);
    x.store(X, up, du4);
    y.store(Y, kDyPitch, kDy);
    if (!STATES) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (row_of(i) < du4) *reinterpret_cast<float4*>(Z + row_of(i) * kDyPitch + tx * 4) = make_float4(z[i][0], z[i][1], z[i][2], z[i][3]);
    }
    __syncthreads();
    if (!STATES) {
      const int i0 = ty * 2;
      float p[2][2] = {};
      const int mine = i0 < n ? du4 : 0;   // (a sequence's last few tokens do not keep every thread)
#pragma unroll 2
      for (int c = 0; c < mine; c += 4) {
        const float4 ua = *reinterpret_cast<const float4*>(U + i0 * up + c), ub = *reinterpret_cast<const float4*>(U + (i0 + 1) * up + c);
        const float4 xa = *reinterpret_cast<const float4*>(X + tx * up + c), xb = *reinterpret_cast<const float4*>(X + (tx + 16) * up + c);
        p[0][0] = fmaf(ua.x, xa.x, fmaf(ua.y, xa.y, fmaf(ua.z, xa.z, fmaf(ua.w, xa.w, p[0][0]))));
        p[0][1] = fmaf(ua.x, xb.x, fmaf(ua.y, xb.y, fmaf(ua.z, xb.z, fmaf(ua.w, xb.w, p[0][1]))));
        p[1][0] = fmaf(ub.x, xa.x, fmaf(ub.y, xa.y, fmaf(ub.z, xa.z, fmaf(ub.w, xa.w, p[1][0]))));
        p[1][1] = fmaf(ub.x, xb.x, fmaf(ub.y, xb.y, fmaf(ub.z, xb.z, fmaf(ub.w, xb.w, p[1][1]))));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + e / 2, j = tx + 16 * (e % 2), away = w.late ? j - i : i - j;
        P[i * kPPitch + j] = away >= 0 ? p[e / 2][e % 2] * power[away] * w.w_near : 0.0f;
      }
      __syncthreads();
      float far[2][4] = {}, near[2][4] = {};
#pragma unroll 2
      for (int c = 0; c < mine; c += 4) {
        const float4 ua = *reinterpret_cast<const float4*>(U + i0 * up + c), ub = *reinterpret_cast<const float4*>(U + (i0 + 1) * up + c);
        const float as[4] = {ua.x, ua.y, ua.z, ua.w}, bs[4] = {ub.x, ub.y, ub.z, ub.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 s = *reinterpret_cast<const float4*>(Z + (c + e) * kDyPitch + tx * 4);
          add4(far[0], as[e], s);
          add4(far[1], bs[e], s);
        }
      }
#pragma unroll 2
      for (int j = 0; j < (i0 < n ? n : 0); j += 4) {
        const float4 pa = *reinterpret_cast<const float4*>(P + i0 * kPPitch + j), pb = *reinterpret_cast<const float4*>(P + (i0 + 1) * kPPitch + j);
        const float as[4] = {pa.x, pa.y, pa.z, pa.w}, bs[4] = {pb.x, pb.y, pb.z, pb.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 v = *reinterpret_cast<const float4*>(Y + (j + e) * kDyPitch + tx * 4);
          add4(near[0], as[e], v);
          add4(near[1], bs[e], v);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int i = i0 + e;
        if (i >= n) continue;
        const float by = power[w.late ? n - 1 - i : i + 1] * w.w_row;
        T* out = static_cast<T*>(w.out) + (int64_t)(token + i) * w.out_ld + (int64_t)h * w.out_head + y0;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (tx * 4 + c < dy) out[tx * 4 + c] = from_float<T>(fmaf(by, far[e][c], near[e][c]));
      }
    }
    // the chunk's own sums first: added one by one to a state of many thousand tokens, terms would lose their last bits
    const float keep = power[n];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k * 64 + ty * 4 >= du4) continue;
      float own[4][4] = {};
#pragma unroll 2
      for (int j = 0; j < n; ++j) {
        const float by = power[w.late ? j + 1 : n - 1 - j] * w.w_x;
        const float4 v = *reinterpret_cast<const float4*>(Y + j * kDyPitch + tx * 4);
        const float4 s = *reinterpret_cast<const float4*>(X + j * up + k * 64 + ty * 4);
        add4(own[0], s.x * by, v);
        add4(own[1], s.y * by, v);
        add4(own[2], s.z * by, v);
        add4(own[3], s.w * by, v);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) z[k * 4 + i][c] = fmaf(keep, z[k * 4 + i][c], own[i][c]);
    }
  }
  if (w.z_out) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int r = row_of(i), col = tx * 4 + c;
        if (r < du && col < dy) w.z_out[at + (int64_t)r * w.dy + y0 + col] = z[i][c];
      }
  }
}

// The parts' own shares, in `z` by item, become the states before each part in the walk's order; the
// state after the last goes to z_out.
struct JoinArgs {
  WalkArgs a;
  float* z[2];               // by item
  const float* z_in[2];      // by sequence; may be NULL
  float* z_out[2];           // by sequence; may be NULL
  int32_t late[2], size;     // size: du dy
};
__global__ void __launch_bounds__(256) k_join(const __grid_constant__ JoinArgs j) {
  pdl_enter();
  const int e = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y % j.a.heads, s = blockIdx.y / j.a.heads, which = blockIdx.z;
  if (e >= j.size) return;
  int first, len;
  sequence_of(j.a, s, first, len);
  const int parts = (len + j.a.part - 1) / j.a.part, base = first / j.a.part + s;
  const float lg = log_decay(j.a.decay, h);
  const int64_t step = (int64_t)j.a.heads * j.size;
  float* z = j.z[which] + base * step + (int64_t)h * j.size + e;
  float state = j.z_in[which] ? j.z_in[which][s * step + (int64_t)h * j.size + e] : 0.0f;
  const float whole = exp2f(j.a.part * lg), last = exp2f((len - (parts - 1) * j.a.part) * lg);
  constexpr int AHEAD = 8;   // (a part's share is written over: the loads of the next few go first)
  for (int t0 = 0; t0 < parts; t0 += AHEAD) {
    float own[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (t0 + i < parts) own[i] = z[(j.late[which] ? parts - 1 - t0 - i : t0 + i) * step];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (t0 + i >= parts) break;
      const int p = j.late[which] ? parts - 1 - t0 - i : t0 + i;
      z[p * step] = state;
      state = fmaf(p == parts - 1 ? last : whole, state, own[i]);
    }
  }
  if (j.z_out[which]) j.z_out[which][s * step + (int64_t)h * j.size + e] = state;
}

// Rows that do not lie on 16 bytes, laid out so that they do, [tokens][heads][dim up to 8], or taken back from there.  A thread moves
// eight elements.
struct PackArgs {
  Heads far[4];
  uint16_t* near[4];
  int32_t dim[4], tokens, heads, seqs;
  const int32_t* seq_start;   // when taken back: rows of no sequence are left as they were
};
template <bool BACK>
__global__ void __launch_bounds__(256) k_pack_heads(const __grid_constant__ PackArgs a) {
  pdl_enter();
  const int which = blockIdx.y, groups = (a.dim[which] + 7) / 8;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, row = e / groups;
  if (row >= (int64_t)a.tokens * a.heads) return;
  const int g = (int)(e - row * groups), h = (int)(row % a.heads);
  const int64_t token = row / a.heads;
  uint16_t* far = static_cast<uint16_t*>(const_cast<void*>(a.far[which].p)) + token * a.far[which].ld + h * a.far[which].head + g * 8;
  uint4* near = reinterpret_cast<uint4*>(a.near[which] + (row * groups + g) * 8);
  const int left = a.dim[which] - g * 8;
  uint32_t w[4];
  if (BACK) {
    if (a.seq_start && (token < a.seq_start[0] || token >= a.seq_start[a.seqs])) return;
    const uint4 v = *near;
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) far[i] = (uint16_t)(i % 2 ? w[i / 2] >> 16 : w[i / 2]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 2 * i < left ? far[2 * i] : 0u, hi = 2 * i + 1 < left ? far[2 * i + 1] : 0u;
      w[i] = lo | hi << 16;
    }
    *near = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The exponent of the largest finite |dout| of each token and head, in f16, for rows on 16 bytes.  WIDTH threads share a row, as many as
// it has pieces of 16 bytes, or more; a thread has a piece of four rows.
template <int WIDTH>
__global__ void __launch_bounds__(256) k_exponents(const Heads dout, int dim, int32_t tokens, uint8_t* tops) {
  pdl_enter();
  constexpr int STEP = 256 / WIDTH, ROWS = 4;
  const int c = threadIdx.x % WIDTH * 8, left = dim - c, h = blockIdx.y;
  const int64_t first = (int64_t)blockIdx.x * (STEP * ROWS) + threadIdx.x / WIDTH;
  const uint16_t* p = static_cast<const uint16_t*>(dout.p) + first * dout.ld + (int64_t)h * dout.head + c;
  uint32_t w[ROWS][4] = {};
#pragma unroll
  for (int i = 0; i < ROWS; ++i, p += STEP * dout.ld) {
    if (first + i * STEP >= tokens) continue;
    if (left >= 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) w[i][e / 2] |= (uint32_t)p[e] << (e % 2 * 16);
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    // (without the sign the bits are in the order of the numbers; those of an infinity or a NaN are above all others)
    const auto most = [&](auto&& of) { return __vmaxu2(__vmaxu2(of(w[i][0]), of(w[i][1])), __vmaxu2(of(w[i][2]), of(w[i][3]))); };
    uint32_t two = most([](uint32_t v) { return v & 0x7FFF7FFFu; });
    if (max(two >> 16, two & 0xFFFFu) >= 0x7C00u)
      two = most([](uint32_t v) {
        v &= 0x7FFF7FFFu;
        return ((v & 0x7C000000u) == 0x7C000000u ? 0u : v & 0xFFFF0000u) | ((v & 0x7C00u) == 0x7C00u ? 0u : v & 0xFFFFu);
      });
#pragma unroll
    for (int d = WIDTH / 2; d; d /= 2) two = __vmaxu2(two, __shfl_xor_sync(0xFFFFFFFFu, two, d));
    const int64_t row = first + i * STEP;
    if (threadIdx.x % WIDTH == 0 && row < tokens) tops[(int64_t)h * tokens + row] = (uint8_t)max(max(two >> 16, two & 0xFFFFu) >> 10, 1u);
  }
}

// ------------------------------------------------------------------ one token
// A block advances one state: warps take its rows in turn, a lane four (or one) of their elements.
template <class T, int N>
__global__ void __launch_bounds__(256) k_attention_step(const __grid_constant__ dgc_attention_one a) {
  pdl_enter();
  __shared__ float part[8][DGC_MAX_HEAD_DIM];
  const int h = blockIdx.x % a.heads, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int64_t r = blockIdx.x / a.heads;
  const int slot = a.slots ? a.slots[r] : (int)r;
  T* out = static_cast<T*>(a.out.data) + r * a.out.ld + (int64_t)h * a.out.head;
  if (slot < 0 || slot >= a.num_slots) {
    for (int c = tid; c < a.value_dim; c += 256) out[c] = from_float<T>(0.0f);
    return;
  }
  const T* q = static_cast<const T*>(a.q.data) + r * a.q.ld + (int64_t)h * a.q.head;
  const T* k = static_cast<const T*>(a.k.data) + r * a.k.ld + (int64_t)h * a.k.head;
  const T* v = static_cast<const T*>(a.v.data) + r * a.v.ld + (int64_t)h * a.v.head;
  float* z = a.state + ((int64_t)slot * a.heads + h) * a.key_dim * a.value_dim;
  const float g = a.decay[h];
  for (int c0 = 0; c0 < a.value_dim; c0 += 32 * N) {
    const int c = c0 + lane * N;
    float vv[N], sum[N] = {};
#pragma unroll
    for (int i = 0; i < N; ++i) vv[i] = c + i < a.value_dim ? to_float<T>(v[c + i]) : 0.0f;
    if (c < a.value_dim) {
      struct alignas(4 * N) Pack { float f[N]; };
      constexpr int ROWS = 8;   // of a lane's loads under way at once (64 x 16 states of 128 x 128: 31 us from DRAM, 23 where L2 holds them)
      for (int d0 = warp; d0 < a.key_dim; d0 += 8 * ROWS) {
        Pack s[ROWS];
        float kk[ROWS], qq[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
          const int d = d0 + 8 * j;
          if (d >= a.key_dim) continue;
          s[j] = *reinterpret_cast<const Pack*>(z + (int64_t)d * a.value_dim + c);
          kk[j] = to_float<T>(k[d]);
          qq[j] = to_float<T>(q[d]);
        }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
          const int d = d0 + 8 * j;
          if (d >= a.key_dim) continue;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            s[j].f[i] = fmaf(g, s[j].f[i], kk[j] * vv[i]);
            sum[i] = fmaf(qq[j], s[j].f[i], sum[i]);
          }
          *reinterpret_cast<Pack*>(z + (int64_t)d * a.value_dim + c) = s[j];
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) part[warp][c + i] = sum[i];
    }
  }
  __syncthreads();
  for (int c = tid; c < a.value_dim; c += 256) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += part[i][c];
    out[c] = from_float<T>(a.scale * sum);
  }
}

// ------------------------------------------------------------------ host
constexpr int kSms = 148;

inline bool bad_heads(const dgc_heads& m, int64_t tokens, size_t es) {
  return m.ld < 0 || m.head < 0 || (tokens > 0 && (!m.data || misaligned(m.data, es)));
}
inline bool bad_output(const dgc_heads& m, int64_t tokens, int64_t heads, int64_t dim, size_t es) {
  if (bad_heads(m, tokens, es)) return true;
  const bool token_major = (heads == 1 || m.head >= dim) && (tokens <= 1 || m.ld >= (heads == 1 ? 0 : (heads - 1) * m.head) + dim);
  const bool head_major = (tokens <= 1 || m.ld >= dim) && (heads == 1 || m.head >= (tokens <= 1 ? 0 : (tokens - 1) * m.ld) + dim);
  return !token_major && !head_major;
}
inline bool bad_dims(int32_t heads, int32_t dk, int32_t dv, float scale) {
  return heads < 1 || heads > 65535 || dk < 1 || dk > DGC_MAX_HEAD_DIM || dv < 1 || dv > DGC_MAX_HEAD_DIM || !std::isfinite(scale);
}
inline bool bad_sizes(const dgc_attention* d) {
  return !d || bad_dtype(d->dtype) || d->num_seqs < 1 || d->tokens < 0 || d->tokens > INT32_MAX - 128 ||
         (!d->seq_start && d->tokens % d->num_seqs != 0) || bad_dims(d->heads, d->key_dim, d->value_dim, d->scale);
}

// Whether tensor copies can fetch the walks' inputs: rows on 16 bytes.  (Heads that share a tensor do not
// move along it, tokens that do are taken by the other kernel.)
inline bool fetched(const Heads& m, int64_t tokens, int64_t heads) {
  return !misaligned(m.p, 16) && (m.ld > 0 || tokens <= 1) && m.ld % 8 == 0 && (m.head % 8 == 0 || heads == 1);
}
inline Heads side(const dgc_heads& m) { return Heads{m.data, m.ld, m.head}; }
// The tensors that are laid out anew in the workspace (q, k, v, dout; out, or dq, dk, dv), and their bytes.  Worth it where the walk in
// 32-bit arithmetic would take a second chunk, and forward in wide heads a little before.  Laid anew and in 32 bits, us, bf16:
//   20 sequences x 12 heads x 125   16 tokens 42, 41 (gradient 114, 82)   24 44, 49 (120, 101)   32 45, 57 (122, 121)   35 46, 72 (124, 154)
//   64 x 16 x 61                    16 69, 49 (171, 107)                  32 75, 64 (181, 150)   40 79, 82 (189, 205)
//   one x 12 x 125                  24 24, 20 (32, 21)                    36 24, 29 (30, 27)     64 24, 33 (30, 33)
struct Laid { int64_t bytes; bool anew[8]; };
inline int dim_of(const dgc_attention* d, int i, bool backward) {
  return i < 2 || (backward && (i == 4 || i == 5)) ? d->key_dim : d->value_dim;
}
inline int64_t laid_bytes(const dgc_attention* d, int dim) { return (d->tokens * d->heads * ((dim + 7) / 8 * 16) + 255) / 256 * 256; }
Laid laid_out(const dgc_attention* d, bool backward) {
  Laid l{};
  const int64_t least = !backward && std::max(d->key_dim, d->value_dim) > 64 ? 20 : 33;   // tokens of a sequence
  if (d->dtype == DGC_F32 || d->tokens < least * d->num_seqs) return l;
  const dgc_heads* all[8] = {&d->q, &d->k, &d->v, &d->dout, backward ? &d->dq : &d->out, &d->dk, &d->dv, nullptr};
  for (int i = 0; i < (backward ? 7 : 5); ++i) {
    if (i == 3 && !backward) continue;
    l.anew[i] = !fetched(side(*all[i]), d->tokens, d->heads);
    if (l.anew[i]) l.bytes += laid_bytes(d, dim_of(d, i, backward));
  }
  return l;
}

// Tokens of a part, 0: sequences are walked whole.  Parts fill SMs that whole sequences would leave idle, but their states come
// first: a walk that takes `states` percent of the rows' time a token (X' in three parts and two of them in heads above 64, 135; 64-wide
// heads 30; 32 bits 90), and two launches (of 16-bit calls the time of 512 tokens); a block's start is counted as `start` tokens.  Of
// one to three parts for each SM the number that ends first, if it ends before whole sequences do.  Of a pack's lengths only the
// mean is known here: its longest is taken to be three times that, and packs of shorter sequences are not cut, since equal ones would
// lose more than uneven ones gain (32 x 4 of 512 on the average x 64 bf16, the longest 4.9 times that: 72, 58 in parts; equal 25, 53).
// Whole and in parts, us: 8 x 16 sequences x heads of 4096 x 64 bf16 118, 149 (of one part each); 24 of 4096 110, 48; 8 of 768 30, 23;
// 36 of 4096 x 128 159, 103 (gradient 175, 261); 2 of 1000 x 128 53, 30; f32, 50 of 1024 x 64 235, 132; 8 of 256 65, 54.
int32_t part_of_call(const dgc_attention* d, bool backward) {
  const int64_t sequences = (int64_t)d->num_seqs * d->heads, units = sequences * (backward ? 3 : 1), len = d->tokens / d->num_seqs;
  const bool uneven = d->seq_start && d->num_seqs > 1;
  if (units >= 2 * kSms || (uneven && len < (d->dtype == DGC_F32 ? 256 : 1024))) return 0;
  const int64_t states = d->dtype == DGC_F32 ? 90 : std::max(d->key_dim, d->value_dim) > 64 ? 135 : 30;
  const int64_t start = d->dtype == DGC_F32 ? 8 : 64;
  const auto rounds = [](int64_t blocks) { return (blocks + kSms - 1) / kSms; };
  int64_t best = 0, ends = rounds(units) * (len * (uneven ? 3 : 1) + start) * 100;
  for (int64_t waves = 1; waves <= 3; ++waves) {
    const int64_t parts = waves * kSms / units;
    if (parts < 1) continue;
    const int64_t part = std::max<int64_t>(128, ((len + parts - 1) / parts + 127) / 128 * 128), cut = (len + part - 1) / part;
    if (cut < (uneven ? 1 : 2)) continue;
    const int64_t end = rounds(cut * units) * (part + start) * 100 + rounds(cut * sequences * (backward ? 2 : 1)) * (part * states + start * 100) +
                        (d->dtype == DGC_F32 ? 0 : 51200);
    if (end < ends) { best = part; ends = end; }
  }
  return (int32_t)best;
}
inline int64_t items_of(const dgc_attention* d, int32_t part) { return part ? d->tokens / part + d->num_seqs : d->num_seqs; }
inline int64_t states_bytes(const dgc_attention* d, int32_t part) {
  return (items_of(d, part) * d->heads * d->key_dim * d->value_dim * 4 + 255) / 256 * 256;
}
// The exponents of dout, which the tensor cores' walk goes by in f16.
inline int64_t tops_bytes(const dgc_attention* d, bool backward) {
  return backward && d->dtype == DGC_F16 && d->tokens > 0 ? (d->tokens * d->heads + 255) / 256 * 256 : 0;
}

template <class T>
int32_t walk(WalkArgs a, int walks, int64_t items, bool states, cudaStream_t s) {
  int du = 0, dy = 0;
  for (int i = 0; i < walks; ++i) { du = std::max(du, a.w[i].du); dy = std::max(dy, a.w[i].dy); }
  a.slices = (dy + kDy - 1) / kDy;
  const int64_t grid = items * a.heads * a.slices;
  if (grid > INT32_MAX) return DGC_EINVAL;
  const dim3 blocks((unsigned)grid, walks);
  const size_t smem = walk_shared(du);
  const int32_t rc = states ? allow_shared<&k_walk<T, true>>(walk_shared(DGC_MAX_HEAD_DIM)) : allow_shared<&k_walk<T, false>>(walk_shared(DGC_MAX_HEAD_DIM));
  if (rc != DGC_OK) return rc;
  if (states) launch(k_walk<T, true>, blocks, kThreads, smem, s, a);
  else launch(k_walk<T, false>, blocks, kThreads, smem, s, a);
  return check_launch();
}

bool on_tensor_cores(const WalkArgs& a, int walks, int32_t dtype, bool states) {
  if (dtype == DGC_F32 || a.tokens == 0) return false;
  for (int i = 0; i < walks; ++i) {
    const Walk& w = a.w[i];
    if (dtype == DGC_F16 && w.dout && !a.dout_tops) return false;
    if ((!states && !fetched(w.u, a.tokens, a.heads)) || !fetched(w.x, a.tokens, a.heads) || !fetched(w.y, a.tokens, a.heads)) return false;
  }
  return true;
}

template <class T, int D, bool STATES>
int32_t walk_tensor(const WalkArgs& a, int walks, int64_t items, cudaStream_t s) {
  TensorWalkArgs g{};
  g.a = a;
  g.a.slices = 1;
  for (int i = 0; i < walks; ++i) {
    const Walk& w = a.w[i];
    const Heads* sides[3] = {&w.u, &w.x, &w.y};
    for (int k = STATES ? 1 : 0; k < 3; ++k) {
      const Heads& m = *sides[k];
      const bool one = m.head == 0 || a.heads == 1;
      const int64_t ld = a.tokens > 1 ? m.ld : 8;
      const int32_t rc = tensor_map(&g.map[i][k], m.p, std::is_same_v<T, __nv_bfloat16>, k == 2 ? w.dy : w.du, a.tokens, one ? 1 : a.heads, ld,
                                    one ? 8 : m.head, kTokens);
      if (rc != DGC_OK) return rc;
      if (one) g.shared[i] |= 1 << k;
    }
    size_t bits = reinterpret_cast<uintptr_t>(w.out) | (a.tokens > 1 ? (size_t)w.out_ld * 2 : 0);
    if (a.heads > 1) bits |= (size_t)w.out_head * 2;
    g.align[i] = bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 2;
  }
  constexpr int exact = std::is_same_v<T, __half> ? 2 : 3;
  bool results = STATES;
  for (int i = 0; i < walks; ++i) results |= a.w[i].z_out != nullptr;
  const auto go = [&](auto parts) {
    constexpr auto kernel = &k_walk_tensor<T, D, STATES, decltype(parts)::value>;
    using L = Layout<D, STATES>;
    const int32_t rc = allow_shared<kernel>(L::shared);
    if (rc != DGC_OK) return rc;
    launch(kernel, dim3((unsigned)(items * a.heads), walks), L::threads, L::shared, s, g);
    return check_launch();
  };
  if constexpr (STATES) return go(std::integral_constant<int, exact>{});
  else return results ? go(std::integral_constant<int, exact>{}) : go(std::integral_constant<int, 2>{});
}
template <class T, bool STATES>
int32_t walk_tensor(const WalkArgs& a, int walks, int64_t items, cudaStream_t s) {
  int dim = 0;
  for (int i = 0; i < walks; ++i) dim = std::max({dim, a.w[i].du, a.w[i].dy});
  return dim <= 64 ? walk_tensor<T, 64, STATES>(a, walks, items, s) : walk_tensor<T, 128, STATES>(a, walks, items, s);
}

int32_t walk(const WalkArgs& a, int32_t dtype, int walks, int64_t items, bool states, cudaStream_t s) {
  if (on_tensor_cores(a, walks, dtype, states)) {
    if (dtype == DGC_BF16)
      return states ? walk_tensor<__nv_bfloat16, true>(a, walks, items, s) : walk_tensor<__nv_bfloat16, false>(a, walks, items, s);
    return states ? walk_tensor<__half, true>(a, walks, items, s) : walk_tensor<__half, false>(a, walks, items, s);
  }
  if (dtype == DGC_F32) return walk<float>(a, walks, items, states, s);
  if (dtype == DGC_BF16) return walk<__nv_bfloat16>(a, walks, items, states, s);
  return walk<__half>(a, walks, items, states, s);
}


int32_t attention(const dgc_attention* d, bool backward, void* stream) {
  if (bad_sizes(d)) return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  if (bad_heads(d->q, d->tokens, es) || bad_heads(d->k, d->tokens, es) || bad_heads(d->v, d->tokens, es) || !d->decay ||
      misaligned(d->decay, 4) || misaligned(d->seq_start, 4) || misaligned(d->s0, 4) || misaligned(d->workspace, 16) ||
      d->workspace_bytes < 0)
    return DGC_EINVAL;
  const auto bad_out = [&](const dgc_heads& m, int32_t dim) { return bad_output(m, d->tokens, d->heads, dim, es); };
  if (backward ? bad_heads(d->dout, d->tokens, es) || bad_out(d->dq, d->key_dim) || bad_out(d->dk, d->key_dim) ||
                     bad_out(d->dv, d->value_dim) || misaligned(d->ds_last, 4) || misaligned(d->ds0, 4)
               : bad_out(d->out, d->value_dim) || misaligned(d->s_last, 4))
    return DGC_EINVAL;
  if (d->tokens == 0 && !(backward ? d->ds0 : d->s_last)) return DGC_OK;
  cudaStream_t s = as_stream(stream);
  const int32_t part = d->workspace ? part_of_call(d, backward) : 0;
  const Laid laid = d->workspace ? laid_out(d, backward) : Laid{};
  const int64_t states = part ? (backward ? 2 : 1) * states_bytes(d, part) : 0;
  const int64_t tops = d->workspace ? tops_bytes(d, backward) : 0;
  if (d->workspace_bytes < states + tops + laid.bytes) return DGC_ECAPACITY;
  const int64_t items = items_of(d, part);
  if (items * d->heads > INT32_MAX / 2) return DGC_EINVAL;
  const int32_t dk = d->key_dim, dv = d->value_dim;
  const float c = d->scale;
  // q, k, v, dout, and out or dq, dk, dv
  Heads t[7] = {side(d->q), side(d->k), side(d->v), side(d->dout), side(backward ? d->dq : d->out), side(d->dk), side(d->dv)};
  const Heads &q = t[0], &k = t[1], &v = t[2], &dout = t[3];
  PackArgs in{}, back{};
  int ins = 0, backs = 0;
  in.tokens = back.tokens = (int32_t)d->tokens;
  in.heads = back.heads = d->heads;
  back.seqs = d->num_seqs;
  back.seq_start = d->seq_start;
  char* to = static_cast<char*>(d->workspace) + states + tops;
  for (int i = 0; i < 7; ++i) {
    if (!laid.anew[i]) continue;
    const int dim = dim_of(d, i, backward), dim8 = (dim + 7) / 8 * 8;
    PackArgs& p = i < 4 ? in : back;
    int& n = i < 4 ? ins : backs;
    p.far[n] = t[i];
    p.near[n] = reinterpret_cast<uint16_t*>(to);
    p.dim[n++] = dim;
    t[i] = Heads{to, (int64_t)d->heads * dim8, dim8};
    to += laid_bytes(d, dim);
  }
  const int64_t blocks = (d->tokens * d->heads * ((std::max(dk, dv) + 7) / 8) + 255) / 256;
  if ((ins || backs) && blocks > INT32_MAX) return DGC_EINVAL;
  if (ins) {
    launch(k_pack_heads<false>, dim3((unsigned)blocks, ins), 256, 0, s, in);
    const int32_t rc = check_launch();
    if (rc != DGC_OK) return rc;
  }
  const auto finish = [&](int32_t rc) {
    if (rc != DGC_OK || !backs) return rc;
    launch(k_pack_heads<true>, dim3((unsigned)blocks, backs), 256, 0, s, back);
    return check_launch();
  };
  const auto at = [](const Heads& m) { return const_cast<void*>(m.p); };
  WalkArgs a{};
  a.decay = d->decay; a.seq_start = d->seq_start; a.tokens = (int32_t)d->tokens; a.seqs = d->num_seqs;
  a.seq_len = (int32_t)(d->tokens / d->num_seqs); a.heads = d->heads; a.part = part;
  a.longest_first = !part && d->seq_start && d->num_seqs > 1 && d->num_seqs <= kSorted && (int64_t)d->num_seqs * d->heads > kSms;
  float* const early = static_cast<float*>(d->workspace);
  float* const late = early + (part ? states_bytes(d, part) / 4 : 0);
  if (tops) {
    uint8_t* const to = static_cast<uint8_t*>(d->workspace) + states;
    a.dout_tops = to;
    if (fetched(dout, d->tokens, d->heads)) {   // (others are walked in 32 bits)
      const int rows = dv <= 64 ? 128 : 64;   // of a block
      const dim3 grid((unsigned)((d->tokens + rows - 1) / rows), (unsigned)d->heads);
      if (dv <= 64) launch(k_exponents<8>, grid, 256, 0, s, dout, dv, a.tokens, to);
      else launch(k_exponents<16>, grid, 256, 0, s, dout, dv, a.tokens, to);
      const int32_t rc = check_launch();
      if (rc != DGC_OK) return rc;
    }
  }
  if (part) {   // the parts' shares of the states, and the states before the parts
    WalkArgs st = a;
    st.w[0] = Walk{{}, k, v, nullptr, 0, 0, nullptr, early, dk, dv, 0, 0, 0.0f, 0.0f, 1.0f, 0};
    if (backward) st.w[1] = Walk{{}, q, dout, nullptr, 0, 0, nullptr, late, dk, dv, 1, 0, 0.0f, 0.0f, c, 0};
    int32_t rc = walk(st, d->dtype, backward ? 2 : 1, items, true, s);
    if (rc != DGC_OK) return rc;
    JoinArgs j{a, {early, late}, {d->s0, d->ds_last}, {backward ? nullptr : d->s_last, d->ds0}, {0, 1}, dk * dv};
    launch(k_join, dim3((dk * dv + 255) / 256, d->num_seqs * d->heads, backward ? 2 : 1), 256, 0, s, j);
    if ((rc = check_launch()) != DGC_OK) return rc;
  }
  const float* const s_in = part ? early : d->s0;
  const float* const e_in = part ? late : d->ds_last;
  if (!backward) {
    a.w[0] = Walk{q, k, v, at(t[4]), t[4].ld, t[4].head, s_in, part ? nullptr : d->s_last, dk, dv, 0, 0, c, c, 1.0f, 0};
    return finish(walk(a, d->dtype, 1, items, false, s));
  }
  a.w[0] = Walk{dout, v, k, at(t[4]), t[4].ld, t[4].head, s_in, nullptr, dv, dk, 0, 1, c, c, 1.0f, 1};
  a.w[1] = Walk{k, q, dout, at(t[6]), t[6].ld, t[6].head, e_in, part ? nullptr : d->ds0, dk, dv, 1, 0, 1.0f, c, c, 0};
  a.w[2] = Walk{v, dout, q, at(t[5]), t[5].ld, t[5].head, e_in, nullptr, dv, dk, 1, 1, 1.0f, c, c, 2};
  return finish(walk(a, d->dtype, 3, items, false, s));
}

}  // namespace

int32_t dgc::attention_waits_out(int* count) { return take_waits_out(count); }

extern "C" {

int32_t dgc_decay_attention_forward(const dgc_attention* a, void* stream) { return attention(a, false, stream); }
int32_t dgc_decay_attention_backward(const dgc_attention* a, void* stream) { return attention(a, true, stream); }

int64_t dgc_decay_attention_workspace_bytes(const dgc_attention* a, int32_t backward) {
  if (bad_sizes(a)) return DGC_EINVAL;
  const int32_t part = part_of_call(a, backward != 0);
  return (part ? (backward ? 2 : 1) * states_bytes(a, part) : 0) + tops_bytes(a, backward != 0) +
         laid_out(a, backward != 0).bytes;
}

int32_t dgc_decay_attention_step(const dgc_attention_one* d, void* stream) {
  if (!d || bad_dtype(d->dtype) || d->rows < 0 || d->num_slots < 0 || bad_dims(d->heads, d->key_dim, d->value_dim, d->scale))
    return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  if (bad_heads(d->q, d->rows, es) || bad_heads(d->k, d->rows, es) || bad_heads(d->v, d->rows, es) ||
      bad_output(d->out, d->rows, d->heads, d->value_dim, es) || misaligned(d->slots, 4) || !d->decay || misaligned(d->decay, 4))
    return DGC_EINVAL;
  if (d->rows == 0) return DGC_OK;
  if (!d->state || misaligned(d->state, 4) || (!d->slots && d->num_slots < d->rows) || (int64_t)d->rows * d->heads > INT32_MAX)
    return DGC_EINVAL;
  const unsigned grid = (unsigned)(d->rows * d->heads);
  cudaStream_t s = as_stream(stream);
  const bool four = d->value_dim % 4 == 0 && !misaligned(d->state, 16);
  if (d->dtype == DGC_F32) four ? launch(k_attention_step<float, 4>, grid, 256, 0, s, *d) : launch(k_attention_step<float, 1>, grid, 256, 0, s, *d);
  else if (d->dtype == DGC_BF16)
    four ? launch(k_attention_step<__nv_bfloat16, 4>, grid, 256, 0, s, *d) : launch(k_attention_step<__nv_bfloat16, 1>, grid, 256, 0, s, *d);
  else four ? launch(k_attention_step<__half, 4>, grid, 256, 0, s, *d) : launch(k_attention_step<__half, 1>, grid, 256, 0, s, *d);
  return check_launch();
}

}  // extern "C"
