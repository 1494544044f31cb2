// The walk of attention.cuh on the tensor cores, for 16-bit types.
//
// A block walks one item of one head in chunks of 128 tokens, with the whole state.  Per chunk four products:
//   P     = U X^T               [128 tokens, 128 tokens]
//   far   = U Z                 [128 tokens, dy]    Z in the type, from shared memory
//   delta = Y^T X'              [dy, du]            X' = X times each token's weight, in parts of the type
//   near  = P' Y                [128 tokens, dy]    P' = P times its weights, in the type, from tensor memory
// and by role:
//   warp 0      brings the tiles of X, U and Y into a ring of slots
//   warp 1      issues the products
//   warps 2-9   keep the state in registers (a thread half a row of Z^T), put it into shared memory, add near
//               and far up and write the rows
//   warps 10-13 make X' and P'
// X' is kept in two parts of the type, in three of bf16 where the state is a result: one would put its rounding, 2^-9,
// into the state, two of 8 bits leave 2^-18.  They are made in the type's own arithmetic: with the weight as w1 + w2 + w3,
//   hi1 = round(x w1), lo1 = x w1 - hi1 (exact, by a multiply-add), and
//   two parts:    hi1, round(x w2 + lo1)
//   three parts:  hi1, s = round(lo1 + hi2), round(x w3 + (what s has lost + lo2))     with hi2 + lo2 = x w2
// which is a third of the instructions that 32-bit products take, taken apart by conversions.  The third part takes the
// place of X, whose product has then been formed.
// f16 has a narrow range.  There a factor (the scale) enters an operand by its significand and a power of two, the rest of it
// the sums, in 32 bits.  And gradients may be far below 1 (a mean loss's are some 1e-5), so that what is as small as they
// are is raised: P and X by a power of two that goes by the largest |dout| of the block's item, which a small kernel has
// looked for, and the gradient's state, as the product takes it, by its own largest element.  (32 sequences of 25000 x 16 x 64,
// backward: 219 -> 259 us, of which the small kernel 12, its results' reading 7, the state's largest 10.  With the largest of
// each chunk's X and U, from their tiles, instead: 278 us, and 103 where 88 are taken forward.)
// dk with a dout of 1e-5 is 4.1e-4 off, where rounding it costs 3.6e-4; 2.8e-3 without.
// The state's sums over a chunk are the tensor core's, over the chunks they are the registers': a tensor core cuts off
// where an addition would round, which over 16 steps does not show and over a long sequence would.
#pragma once

#include <cfloat>

#include "attention.cuh"
#include "tensor.cuh"

namespace dgc {

constexpr int kTokens = 128;

struct TensorWalkArgs {
  CUtensorMap map[kMaxWalks][3];   // u, x, y: [heads][tokens][dim]
  WalkArgs a;
  int32_t shared[kMaxWalks];       // bit i: the heads share u, x or y
  int32_t align[kMaxWalks];        // bytes the output's rows are aligned to: 32, 16 or 2
};

// How a block's shared memory and warps are dealt out.  Of 128 x 128 tiles there is room for seven: X' in two parts (a third
// takes the place of X, whose product has then been formed), the state and four slots.  Walks that write no rows have
// two X', the one made while the other is multiplied, and twice the warps that make it (states of 2 x 65536 x 16 x 128: 508 -> 394 us).
template <int D, bool STATES> struct Layout {
  static constexpr int slot_bytes = kTokens * D * 2, sets = STATES ? 2 : 1, slots = D == 64 ? 8 : STATES ? 3 : 4;
  static constexpr int makers = STATES ? 8 : 4, threads = (10 + makers) * 32;
  static constexpr int shared = 1024 + (slots + sets * 2) * slot_bytes + (STATES ? 0 : D * D * 2);
};

__device__ __forceinline__ void store_shared(uint32_t at, const uint32_t (&w)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
__device__ __forceinline__ void load_shared(uint32_t at, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
}

// 2^x where it stands: kept from chunk to chunk, the values would not fit the registers.
__device__ __forceinline__ float exp2_here(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(127 + k) << 23); }   // -126 .. 127
// 2^to over the power of two in `bits`, a 32-bit number >= 0, and its inverse; both normal numbers.
struct Raise { float up, down; };
__device__ __forceinline__ Raise raise_to(int to, uint32_t bits) {
  const int k = max(min(to + 127 - (int)(bits >> 23), 126), -126);
  return Raise{power_of_two(k), power_of_two(-k)};
}
// A factor w of an operand as it enters the product, and what is left of it for the sums, in 32 bits.
struct Factor { float by, back; };
__device__ __forceinline__ float kept_finite(float v) { return fminf(fmaxf(v, -FLT_MAX), FLT_MAX); }
// w's significand, in [1, 2) (less below 2^-126), times 2^up.
__device__ __forceinline__ float power_in(float w) { return __uint_as_float(max(__float_as_uint(w) & 0x7F800000u, 0x00800000u)); }
__device__ __forceinline__ Factor factor_of(float w, int up) {
  return Factor{w / power_in(w) * power_of_two(up), kept_finite(power_in(w) * power_of_two(-up))};
}
template <int ID, int THREADS>
__device__ __forceinline__ void meet() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory"); }
// The largest |v|, four at a time; a NaN is passed over.
template <int N>
__device__ __forceinline__ float largest(const float (&v)[N]) {
  float top[4] = {};
#pragma unroll
  for (int i = 0; i < N; i += 8)
#pragma unroll
    for (int k = 0; k < 4; ++k) top[k] = fmaxf(fmaxf(top[k], fabsf(v[i + k])), fabsf(v[i + 4 + k]));
  return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}

template <class T, int D, bool STATES, int PARTS>
__global__ void __launch_bounds__(Layout<D, STATES>::threads, 1) k_walk_tensor(const __grid_constant__ TensorWalkArgs g) {
  constexpr bool BF16 = std::is_same_v<T, __nv_bfloat16>, RAISED = !BF16;   // RAISED: powers of two keep the operands in range
  using L = Layout<D, STATES>;
  constexpr int SLOTS = L::slots, SLOT = L::slot_bytes, NB = L::sets, MAKERS = L::makers, BOX = kTokens * 128, PER = STATES ? 2 : 3;
  constexpr uint32_t P_AT = 0, NEAR = 128, FAR = 128 + D, DELTA = 128 + 2 * D;
  extern __shared__ char dynamic[];
  __shared__ __align__(8) uint64_t bars[2 * 8 + 12];
  __shared__ __align__(16) uint32_t z_tops[2][8], warp_tops[L::threads / 32];   // what each warp has seen: of the state (two chunks'), of dout
  __shared__ float power[kTokens + 1];   // g^0 .. g^128
  __shared__ uint32_t tmem_at;
  __shared__ volatile int failed;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t ring = (shared_u32(dynamic) + 1023) & ~1023u, scaled = ring + SLOTS * SLOT, zs = scaled + NB * 2 * SLOT;
  const auto full = [&](int i) { return shared_u32(bars + i % SLOTS); };
  const auto empty = [&](int i) { return shared_u32(bars + 8 + i % SLOTS); };
  const auto tile = [&](int i) { return ring + i % SLOTS * SLOT; };
  const uint32_t p_full = shared_u32(bars + 16), p_ready = p_full + 8, o_full = p_full + 16, o_empty = p_full + 24, x_ready = p_full + 80,
                 d_full = p_full + 40, z_ready = p_full + 48, z_empty = p_full + 56, d_empty = p_full + 32, x_free = p_full + 64;
  if (tid == 0) {
    failed = 0;
    for (int s = 0; s < SLOTS; ++s) { barrier_init(shared_u32(bars + s), 1); barrier_init(shared_u32(bars + 8 + s), 1); }
    barrier_init(p_full, 1); barrier_init(p_ready, 4); barrier_init(o_full, 1); barrier_init(o_empty, 8);
    for (int b = 0; b < 2; ++b) { barrier_init(x_ready + b * 8, MAKERS); barrier_init(x_free + b * 8, 1); }
    barrier_init(d_full, 1); barrier_init(d_empty, 8); barrier_init(z_ready, 8); barrier_init(z_empty, 1);
    barrier_init_visible();
  }
  if (warp == 1) tmem_alloc<1>(shared_u32(&tmem_at), 512);
  pdl_enter();
  const int which = blockIdx.y, h = blockIdx.x % g.a.heads, item = blockIdx.x / g.a.heads;
  const Walk& w = g.a.w[which];
  const Item it = item_of(g.a, item);
  const float lg = log_decay(g.a.decay, h);
  if (tid <= kTokens) power[tid] = exp2f(tid * lg);
  if (RAISED && w.dout) {   // the exponent of the item's largest dout
    const uint8_t* from = g.a.dout_tops + (int64_t)h * g.a.tokens + it.first;
    uint32_t top = 1;
#pragma unroll 4
    for (int i = tid; i < it.len; i += L::threads) top = max(top, (uint32_t)from[i]);
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (lane == 0) warp_tops[warp] = top;
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;
  const int chunks = (it.len + kTokens - 1) / kTokens;
  const bool late = w.late;
  Factor x_is{w.w_x, 1.0f}, near_is{w.w_near, 1.0f};
  if constexpr (RAISED) {
    // without a gradient: X by less than 1, and P by w_near, of a scale within 2^-12 .. 2^15
    int x_up = fabsf(w.w_x) > power_in(w.w_x) ? -1 : 0, near_up = min(max((int)(__float_as_uint(w.w_near) >> 23 & 255) - 127, -12), 14);
    if (w.dout) {
      uint32_t top = 0;
      for (int i = 0; i < L::threads / 32; ++i) top = max(top, warp_tops[i]);
      const int e = (int)top - 15;
      near_up = max(near_up, -2 - e - (32 - __clz(w.du - 1)));   // |P| < du 2^(e + 1) 2^16, and its factor's significand 2
      if (w.dout == 2) x_up = min(13 - e, 14);                   // X' < 2^15
    }
    x_is = factor_of(w.w_x, x_up);
    near_is = factor_of(w.w_near, near_up);
  }
  const auto first_of = [&](int c) { return (late ? chunks - 1 - c : c) * kTokens; };
  bool ok = true;

  if (warp == 0) {
    if (elect_one()) {
      for (int i = 0; i < chunks * PER && ok; ++i) {
        const int part = i % PER, side = STATES ? part + 1 : part;   // u, x, y in turn: the order in which slots come free
        if (!(ok = wait_for(empty(i), (i / SLOTS & 1) ^ 1, &failed))) break;
        arrive_expect(full(i), SLOT);
        const int z = g.shared[which] >> side & 1 ? 0 : h, y = it.first + first_of(i / PER);
#pragma unroll
        for (int b = 0; b < D / 64; ++b) load_tile<1>(tile(i) + b * BOX, &g.map[which][side], full(i), b * 64, y, z);
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t p_what = product_descriptor(128, 128, BF16, false, false), far_what = product_descriptor(128, D, BF16, false, false),
                         near_what = product_descriptor(128, D, BF16, false, true), d_what = product_descriptor(128, D, BF16, true, true);
      const auto there = [&](int i) { return wait_for(full(i), i / SLOTS & 1, &failed); };
      const auto form_p = [&](int c) {
        const int ui = c * PER, xi = ui + 1;
        if (!there(ui) || !there(xi)) return false;
        fence_after();
        const uint64_t u = tile_descriptor(tile(ui), 16), x = tile_descriptor(tile(xi), 16);
#pragma unroll 1
        for (int k = 0; k < D / 16; ++k)
          product<1>(tmem + P_AT, u + (k / 4 * BOX + k % 4 * 32) / 16, x + (k / 4 * BOX + k % 4 * 32) / 16, p_what, k > 0);
        commit<1>(p_full);
        return true;
      };
      if (!STATES && chunks > 0) ok = form_p(0);
      for (int c = 0; c < chunks && ok; ++c) {
        const int xi = c * PER + PER - 2, yi = xi + 1;
        if (!STATES) {
          if (!(ok = wait_for(z_ready, c & 1, &failed) && wait_for(o_empty, (c & 1) ^ 1, &failed))) break;
          fence_after();
          const uint64_t u = tile_descriptor(tile(xi - 1), 16), z = tile_descriptor(zs, 16);
#pragma unroll 1
          for (int k = 0; k < D / 16; ++k)
            product<1>(tmem + FAR, u + (k / 4 * BOX + k % 4 * 32) / 16, z + (k / 4 * (D * 128) + k % 4 * 32) / 16, far_what, k > 0);
          commit<1>(empty(xi - 1));
          commit<1>(z_empty);
        }
        if (!(ok = there(yi) && wait_for(x_ready + c % NB * 8, c / NB & 1, &failed) && wait_for(d_empty, (c & 1) ^ 1, &failed))) break;
        fence_after();
        const uint64_t y = tile_descriptor(tile(yi), BOX), xh = tile_descriptor(scaled + c % NB * 2 * SLOT, BOX), xl = xh + SLOT / 16;
#pragma unroll 1
        for (int k = 0; k < kTokens / 16; ++k) product<1>(tmem + DELTA, y + k * 128, xh + k * 128, d_what, k > 0);
#pragma unroll 1
        for (int k = 0; k < kTokens / 16; ++k) product<1>(tmem + DELTA, y + k * 128, xl + k * 128, d_what, true);
        if (PARTS == 3) {
          const uint64_t xr = tile_descriptor(tile(xi), BOX);
#pragma unroll 1
          for (int k = 0; k < kTokens / 16; ++k) product<1>(tmem + DELTA, y + k * 128, xr + k * 128, d_what, true);
        }
        commit<1>(d_full);
        commit<1>(x_free + c % NB * 8);
        commit<1>(empty(xi));
        if (!STATES) {
          if (!(ok = wait_for(p_ready, c & 1, &failed))) break;
          fence_after();
#pragma unroll 1
          for (int k = 0; k < kTokens / 16; ++k) product_tmem(tmem + NEAR, tmem + P_AT + k * 8, y + k * 128, near_what, k > 0);
          commit<1>(o_full);
        }
        commit<1>(empty(yi));
        if (!STATES && c + 1 < chunks) ok = form_p(c + 1);
      }
    }
  } else if (warp < 10) {
    constexpr int H = D / 2;
    const int quad = warp % 4, half = (warp - 2) / 4, r = quad * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + half * H;
    const int64_t at = ((int64_t)(g.a.part ? item : it.s) * g.a.heads + h) * w.du * w.dy;
    float z[H];
#pragma unroll
    for (int d = 0; d < H; ++d) {
      const int u = half * H + d;
      z[d] = !STATES && w.z_in && r < w.dy && u < w.du ? w.z_in[at + (w.turned ? r * w.du + u : u * w.dy + r)] : 0.0f;
    }
    float z_back = 1.0f;
    // The state before chunk c, as the product takes it.  (All of these warps come here for every chunk, those that have given
    // up, too: they meet at a barrier that does not count time.)
    const auto show = [&](int c) {
      float up = 1.0f;
      if (RAISED && late) {   // (the gradient's state is as small as dout is)
        uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, r < w.dy ? __float_as_uint(largest(z)) : 0u);
        if (lane == 0) z_tops[c & 1][warp - 2] = bits;
        meet<2, 256>();
        const uint4 a = *reinterpret_cast<const uint4*>(z_tops[c & 1]), b = *reinterpret_cast<const uint4*>(z_tops[c & 1] + 4);
        bits = max(max(max(a.x, a.y), max(a.z, a.w)), max(max(b.x, b.y), max(b.z, b.w)));
        const Raise raise = raise_to(14, bits);
        up = raise.up;
        z_back = raise.down;
      }
      if (!ok) return;
      if (r < D) {
#pragma unroll
        for (int d = 0; d < H; d += 8) {
          const int u = half * H + d;
          uint32_t p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            Val<2> two{{z[d + 2 * e], z[d + 2 * e + 1]}};
            if (RAISED) two = mul_(two, fill<2>(up));
            p[e] = pack<T, 2>(two.v);
          }
          store_shared(zs + u / 64 * (D * 128) + r * 128 + (((u % 64 / 8) ^ (r & 7)) << 4), p);
        }
      }
      shared_to_async();
      __syncwarp();
      if (lane == 0) arrive(z_ready);
    };
    if (!STATES && chunks > 0) show(0);
    for (int c = 0; c < chunks; ++c) {
      const int from = first_of(c), n = min(kTokens, it.len - from);
      if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(d_full, c & 1, &failed));
      if (ok) {
        fence_after();
        const float keep = power[n], back = RAISED && late ? x_is.back * power[1] : x_is.back;
#pragma unroll
        for (int b = 0; b < H; b += 16) {
          uint32_t v[16];
          tmem_ld16(lanes + DELTA + b, v);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            Val<2> own{{__uint_as_float(v[e]), __uint_as_float(v[e + 1])}};
            if (RAISED) own = mul_(own, fill<2>(back));
            const Val<2> now = fma_(fill<2>(keep), Val<2>{{z[b + e], z[b + e + 1]}}, own);
            z[b + e] = now.v[0];
            z[b + e + 1] = now.v[1];
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(d_empty);
      }
      if (STATES) continue;
      const float far_back = z_back;
      if (c + 1 < chunks) {
        if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(z_empty, c & 1, &failed));
        show(c + 1);
      }
      if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(o_full, c & 1, &failed));
      if (!ok) continue;
      fence_after();
      const bool there = r < n;
      float by = there ? power[late ? n - 1 - r : r + 1] * w.w_row : 0.0f;
      if (RAISED) by = kept_finite(by * far_back);
      T* out = static_cast<T*>(w.out) + (int64_t)(it.first + from + r) * w.out_ld + (int64_t)h * w.out_head + half * H;
#pragma unroll 1
      for (int b = 0; b < H; b += 16) {
        uint32_t x[16], y[16], packed[8];
        tmem_ld16(lanes + FAR + b, x);
        tmem_ld16(lanes + NEAR + b, y);
        tmem_wait_ld();
        if (b + 16 == H) {
          fence_before();
          __syncwarp();
          if (lane == 0) arrive(o_empty);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          Val<2> near{{__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])}};
          if (RAISED) near = mul_(near, fill<2>(near_is.back));
          const Val<2> v = fma_(Val<2>{{__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])}}, fill<2>(by), near);
          packed[e] = pack<T, 2>(v.v);
        }
        const int left = w.dy - half * H - b;
        if (!there) continue;
        if (g.align[which] == 32 && left >= 16) {
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + b), DGC_I8(packed, 0) : "memory");
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (g.align[which] >= 16 && left >= 8 * e + 8) {
              *reinterpret_cast<uint4*>(out + b + 8 * e) = make_uint4(packed[4 * e], packed[4 * e + 1], packed[4 * e + 2], packed[4 * e + 3]);
            } else {
#pragma unroll
              for (int f = 0; f < 8; ++f)
                if (8 * e + f < left)
                  store_word<T, 1>(out + b + 8 * e + f, f % 2 ? packed[4 * e + f / 2] >> 16 : packed[4 * e + f / 2] & 0xFFFFu);
            }
          }
        }
      }
    }
    if (w.z_out && ok && r < w.dy && !(STATES && it.len == 0)) {
      float* to = w.z_out + at + (int64_t)half * H * w.dy + r;
#pragma unroll
      for (int d = 0; d < H; ++d, to += w.dy)
        if (half * H + d < w.du) *to = z[d];
    }
  } else {
    const int quad = warp % 4, i = quad * 32 + lane, t = (warp - 10) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + P_AT;
    // the weights of the tokens that this thread meets in X, in a chunk that is whole
    struct Weight { uint32_t part[PARTS]; };
    const auto weight_of = [&](int j, int n) {
      float v = power[late ? RAISED ? j : j + 1 : n - 1 - j] * x_is.by;   // (RAISED: the decay that all of a late walk's have enters in 32 bits)
      Weight r;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const float both[2] = {v, v};
        r.part[p] = pack<T, 2>(both);
        float kept[2];
        unpack<T, 2>(r.part[p], kept);
        v -= kept[0];
      }
      return r;
    };
    constexpr int STEP = MAKERS * 4, MET = kTokens / STEP;   // from one token that a thread meets to the next
    Weight token[MET];
#pragma unroll
    for (int e = 0; e < MET; ++e) token[e] = weight_of(e * STEP + t / 8, kTokens);
    const float twice = power[2];
    for (int c = 0; c < chunks; ++c) {
      const int xi = c * PER + PER - 2, yi = xi + 1, n = min(kTokens, it.len - first_of(c));
      if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(full(xi), xi / SLOTS & 1, &failed));
      if (ok && n < kTokens) ok = __all_sync(0xFFFFFFFFu, wait_for(full(yi), yi / SLOTS & 1, &failed));
      if (ok && PARTS == 3 && !STATES) ok = __all_sync(0xFFFFFFFFu, wait_for(p_full, c & 1, &failed));   // (X is read no more)
      const uint32_t hi = scaled + c % NB * 2 * SLOT, lo = hi + SLOT;
      if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(x_free + c % NB * 8, (c / NB & 1) ^ 1, &failed));
      if (!ok) break;
      const auto scale = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
        for (int i0 = 0; i0 < SLOT / 16 / (MAKERS * 32); i0 += 4) {
          constexpr int STRIDE = MAKERS * 32 * 16;
          uint32_t x[4][4];
#pragma unroll
          for (int k = 0; k < 4; ++k) load_shared(tile(xi) + (i0 + k) * STRIDE + t * 16, x[k]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t off = (i0 + k) * STRIDE + t * 16;
            const int j = (i0 + k) % MET * STEP + t / 8;
            const bool there = WHOLE || j < n;   // (what lies behind the sequence may be anything)
            Weight by = token[(i0 + k) % MET];
            if (!WHOLE) by = weight_of(j, there ? n : kTokens);
            uint32_t part[3][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t v = there ? x[k][e] : 0u;
              const uint32_t hi1 = mul16<T>(v, by.part[0]), lo1 = fma16<T>(v, by.part[0], hi1 ^ 0x80008000u);
              part[0][e] = hi1;
              if constexpr (PARTS == 2) {
                part[1][e] = fma16<T>(v, by.part[1], lo1);
              } else {
                const uint32_t hi2 = mul16<T>(v, by.part[1]), lo2 = fma16<T>(v, by.part[1], hi2 ^ 0x80008000u);
                const uint32_t s = add16<T>(lo1, hi2), back = sub16<T>(s, lo1);
                const uint32_t lost = add16<T>(sub16<T>(lo1, sub16<T>(s, back)), sub16<T>(hi2, back));
                part[1][e] = s;
                part[2][e] = fma16<T>(v, by.part[2], add16<T>(lost, lo2));
              }
            }
            store_shared(hi + off, part[0]);
            store_shared(lo + off, part[1]);
            if (PARTS == 3) store_shared(tile(xi) + off, part[2]);
          }
        }
      };
      if (n == kTokens) {
        scale(std::true_type{});
      } else {
        scale(std::false_type{});
        const uint32_t none[4] = {};
        for (int e = n * 8 + t; e < kTokens * 8; e += MAKERS * 32)
#pragma unroll
          for (int b = 0; b < D / 64; ++b) store_shared(tile(yi) + b * BOX + e * 16, none);
      }
      shared_to_async();
      __syncwarp();
      if (lane == 0) arrive(x_ready + c % NB * 8);
      if (STATES) continue;
      if (!(ok = __all_sync(0xFFFFFFFFu, wait_for(p_full, c & 1, &failed)))) break;
      fence_after();
      const int j_first = late ? i : 0, j_span = (late ? n - 1 : i) - j_first;   // the columns that count
      // P' takes the place of columns of P that have been read; the next are on their way meanwhile
      const auto weigh = [&](int b, const uint32_t (&v)[32]) {
        uint32_t packed[16] = {};
        if (late ? b >= quad && b * 32 < n : b <= quad) {
          if (late ? b > quad && b * 32 + 32 <= n : b < quad) {
            // all count: a column's weight is its neighbour's times the decay, from the nearest on
            const float near1 = power[late ? b * 32 - i : i - 31 - b * 32] * near_is.by, near2 = near1 * power[1];
            Val<2> by = late ? Val<2>{{near1, near2}} : Val<2>{{near2, near1}};
            if (late) {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const Val<2> p = mul_(Val<2>{{__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])}}, by);
                packed[e] = pack<T, 2>(p.v);
                by = mul_(by, fill<2>(twice));
              }
            } else {
#pragma unroll
              for (int e = 15; e >= 0; --e) {
                const Val<2> p = mul_(Val<2>{{__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])}}, by);
                packed[e] = pack<T, 2>(p.v);
                by = mul_(by, fill<2>(twice));
              }
            }
          } else {
            const float step = late ? lg : -lg, start = (late ? b * 32 - i : i - b * 32) * lg;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float p[2];
#pragma unroll
              for (int f = 0; f < 2; ++f) {
                const int j = 2 * e + f;
                const float q = __uint_as_float(v[j]) * near_is.by * exp2_here(fmaf(j, step, start));
                p[f] = (unsigned)(b * 32 + j - j_first) <= (unsigned)j_span && j_span >= 0 ? q : 0.0f;
              }
              packed[e] = pack<T, 2>(p);
            }
          }
        }
        tmem_st16(lanes + b * 16, packed);
      };
      uint32_t even[32], odd[32];
      tmem_ld32(lanes, even);
#pragma unroll 1
      for (int b = 0; b < 4; b += 2) {
        tmem_wait_ld();
        tmem_ld32(lanes + b * 32 + 32, odd);
        weigh(b, even);
        tmem_wait_ld();
        if (b < 2) tmem_ld32(lanes + b * 32 + 64, even);
        weigh(b + 1, odd);
      }
      tmem_wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(p_ready);
    }
  }
  fence_before();
  __syncthreads();
  if (failed) let_copies_end();
  fence_after();
  if (warp == 1) tmem_free<1>(tmem, 512);
}

}  // namespace dgc
