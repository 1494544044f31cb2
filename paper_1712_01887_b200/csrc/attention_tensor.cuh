// The walk of attention.cuh on the tensor cores, for 16-bit types.
//
// A block walks one item of one head in chunks of 128 tokens, with the whole state.  Per chunk four products:
//   P     = U X^T               [128 tokens, 128 tokens]
//   far   = U Z                 [128 tokens, dy]    Z in the type, from shared memory
//   delta = Y^T X'              [dy, du]            X' = X times each token's weight, in two parts of the type
//   near  = P' Y                [128 tokens, dy]    P' = P times its weights, in the type, from tensor memory
// and by role:
//   warp 0      brings the tiles of X, U and Y into a ring of slots
//   warp 1      issues the products
//   warps 2-5   make X' (the rounding of x g^n to one part would be the state's: 2^-9 of it, where the state is a
//               result in 32 bits), keep the state in registers (a thread a row of Z^T), and put it into shared memory
//   warps 6-9   make P', add near and far up and write the rows
// The state's sums over a chunk are the tensor core's, over the chunks they are the registers': a tensor core cuts off
// where an addition would round, which over 16 steps does not show and over a long sequence would.
#pragma once

#include "attention.cuh"
#include "tensor.cuh"

namespace dgc {

constexpr int kTokens = 128, kTensorThreads = 320;

struct TensorWalkArgs {
  CUtensorMap map[kMaxWalks][3];   // u, x, y: [heads][tokens][dim]
  WalkArgs a;
  int32_t shared[kMaxWalks];       // bit i: the heads share u, x or y
  int32_t align[kMaxWalks];        // bytes the output's rows are aligned to: 32, 16 or 2
};

template <int D, bool STATES> constexpr int kSlots = D == 128 ? (STATES ? 5 : 4) : 8;
template <int D> constexpr int kSlotBytes = kTokens * D * 2;
template <int D, bool STATES> constexpr int kTensorShared = 1024 + (kSlots<D, STATES> + 2) * kSlotBytes<D> + (STATES ? 0 : D * D * 2);

__device__ __forceinline__ void store_shared(uint32_t at, const uint32_t (&w)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}

template <class T, int D, bool STATES>
__global__ void __launch_bounds__(kTensorThreads, 1) k_walk_tensor(const __grid_constant__ TensorWalkArgs g) {
  constexpr int SLOTS = kSlots<D, STATES>, SLOT = kSlotBytes<D>, BOX = kTokens * 128, PER = STATES ? 2 : 3;
  constexpr bool BF16 = std::is_same_v<T, __nv_bfloat16>;
  constexpr uint32_t P_AT = 0, NEAR = 128, FAR = 128 + D, DELTA = 128 + 2 * D;
  extern __shared__ char dynamic[];
  __shared__ __align__(8) uint64_t bars[2 * 8 + 8];
  __shared__ float power[kTokens + 1];   // g^0 .. g^128
  __shared__ uint32_t tmem_at;
  __shared__ volatile int failed;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t ring = (shared_u32(dynamic) + 1023) & ~1023u, hi = ring + SLOTS * SLOT, lo = hi + SLOT, zs = lo + SLOT;
  const auto full = [&](int i) { return shared_u32(bars + i % SLOTS); };
  const auto empty = [&](int i) { return shared_u32(bars + 8 + i % SLOTS); };
  const auto tile = [&](int i) { return ring + i % SLOTS * SLOT; };
  const uint32_t p_full = shared_u32(bars + 16), p_ready = p_full + 8, o_full = p_full + 16, o_empty = p_full + 24, x_ready = p_full + 32,
                 d_full = p_full + 40, z_ready = p_full + 48, z_empty = p_full + 56;
  if (tid == 0) {
    failed = 0;
    for (int s = 0; s < SLOTS; ++s) { barrier_init(shared_u32(bars + s), 1); barrier_init(shared_u32(bars + 8 + s), 1); }
    barrier_init(p_full, 1); barrier_init(p_ready, 4); barrier_init(o_full, 1); barrier_init(o_empty, 4);
    barrier_init(x_ready, 4); barrier_init(d_full, 1); barrier_init(z_ready, 4); barrier_init(z_empty, 1);
    barrier_init_visible();
  }
  if (warp == 1) tmem_alloc<1>(shared_u32(&tmem_at), 512);
  pdl_enter();
  const int which = blockIdx.y, h = blockIdx.x % g.a.heads, item = blockIdx.x / g.a.heads;
  const Walk& w = g.a.w[which];
  const Item it = item_of(g.a, item);
  const float lg = log_decay(g.a.decay, h);
  if (tid <= kTokens) power[tid] = exp2f(tid * lg);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;
  const int chunks = (it.len + kTokens - 1) / kTokens;
  const bool late = w.late;
  const auto first_of = [&](int c) { return (late ? chunks - 1 - c : c) * kTokens; };
  bool ok = true;

  if (warp == 0) {
    if (elect_one()) {
      for (int i = 0; i < chunks * PER && ok; ++i) {
        const int part = i % PER, side = STATES ? part + 1 : part == 0 ? 1 : part == 1 ? 0 : 2;   // x, u, y in turn
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
      for (int c = 0; c < chunks; ++c) {
        const int xi = c * PER, ui = xi + 1, yi = xi + PER - 1;
        const auto there = [&](int i) { return wait_for(full(i), i / SLOTS & 1, &failed); };
        if (!there(xi)) break;
        if (!STATES) {
          if (!there(ui)) break;
          fence_after();
          const uint64_t u = tile_descriptor(tile(ui), 16), x = tile_descriptor(tile(xi), 16), z = tile_descriptor(zs, 16);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            product<1>(tmem + P_AT, u + (k / 4 * BOX + k % 4 * 32) / 16, x + (k / 4 * BOX + k % 4 * 32) / 16, p_what, k > 0);
          commit<1>(p_full);
          if (!wait_for(z_ready, c & 1, &failed) || !wait_for(o_empty, (c & 1) ^ 1, &failed)) break;
          fence_after();
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            product<1>(tmem + FAR, u + (k / 4 * BOX + k % 4 * 32) / 16, z + (k / 4 * (D * 128) + k % 4 * 32) / 16, far_what, k > 0);
          commit<1>(empty(ui));
          commit<1>(z_empty);
        }
        if (!there(yi) || !wait_for(x_ready, c & 1, &failed)) break;
        fence_after();
        const uint64_t y = tile_descriptor(tile(yi), BOX), xh = tile_descriptor(hi, BOX), xl = tile_descriptor(lo, BOX);
#pragma unroll
        for (int k = 0; k < kTokens / 16; ++k) product<1>(tmem + DELTA, y + k * 128, xh + k * 128, d_what, k > 0);
#pragma unroll
        for (int k = 0; k < kTokens / 16; ++k) product<1>(tmem + DELTA, y + k * 128, xl + k * 128, d_what, true);
        commit<1>(d_full);
        commit<1>(empty(xi));
        if (STATES) {
          commit<1>(empty(yi));
        } else {
          if (!wait_for(p_ready, c & 1, &failed)) break;
          fence_after();
#pragma unroll
          for (int k = 0; k < kTokens / 16; ++k) product_tmem(tmem + NEAR, tmem + P_AT + k * 8, y + k * 128, near_what, k > 0);
          commit<1>(o_full);
          commit<1>(empty(yi));
        }
      }
    }
  } else if (warp < 6) {
    const int quad = warp % 4, r = quad * 32 + lane, t = (warp - 2) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + DELTA;
    const int64_t at = ((int64_t)(g.a.part ? item : it.s) * g.a.heads + h) * w.du * w.dy;
    float z[D];
#pragma unroll
    for (int d = 0; d < D; ++d)
      z[d] = !STATES && w.z_in && r < w.dy && d < w.du ? w.z_in[at + (w.turned ? r * w.du + d : d * w.dy + r)] : 0.0f;
    const auto show = [&] {   // the state, as the product takes it
      if (r < D) {
#pragma unroll
        for (int d = 0; d < D; d += 8) {
          uint32_t p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float two[2] = {z[d + 2 * e], z[d + 2 * e + 1]};
            p[e] = pack<T, 2>(two);
          }
          store_shared(zs + d / 64 * (D * 128) + r * 128 + (((d % 64 / 8) ^ (r & 7)) << 4), p);
        }
      }
      shared_to_async();
      __syncwarp();
      if (lane == 0) arrive(z_ready);
    };
    if (!STATES && chunks > 0) show();
    for (int c = 0; c < chunks; ++c) {
      const int xi = c * PER, yi = xi + PER - 1, n = min(kTokens, it.len - first_of(c));
      ok = __all_sync(0xFFFFFFFFu, wait_for(full(xi), xi / SLOTS & 1, &failed));
      if (ok && n < kTokens) ok = __all_sync(0xFFFFFFFFu, wait_for(full(yi), yi / SLOTS & 1, &failed));
      if (!ok) break;
#pragma unroll 4
      for (int i = 0; i < SLOT / 16 / 128; ++i) {
        const uint32_t off = (i * 128 + t) * 16;
        const int j = off / 128 % kTokens;
        const float by = j < n ? power[late ? j + 1 : n - 1 - j] * w.w_x : 0.0f;
        uint32_t x[4], ph[4], pl[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(tile(xi) + off));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[2], top[2], rest[2];
          unpack<T, 2>(x[e], v);
          v[0] = j < n ? v[0] * by : 0.0f;   // (what lies behind the sequence may be anything)
          v[1] = j < n ? v[1] * by : 0.0f;
          ph[e] = pack<T, 2>(v);
          unpack<T, 2>(ph[e], top);
          rest[0] = v[0] - top[0];
          rest[1] = v[1] - top[1];
          pl[e] = pack<T, 2>(rest);
        }
        store_shared(hi + off, ph);
        store_shared(lo + off, pl);
      }
      if (n < kTokens) {
        const uint32_t none[4] = {};
        for (int i = n * 8 + t; i < kTokens * 8; i += 128)
#pragma unroll
          for (int b = 0; b < D / 64; ++b) store_shared(tile(yi) + b * BOX + i * 16, none);
      }
      shared_to_async();
      __syncwarp();
      if (lane == 0) arrive(x_ready);
      if (!(ok = __all_sync(0xFFFFFFFFu, wait_for(d_full, c & 1, &failed)))) break;
      fence_after();
      const float keep = power[n];
#pragma unroll
      for (int b = 0; b < D; b += 32) {
        uint32_t v[32];
        tmem_ld32(lanes + b, v);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; ++e) z[b + e] = fmaf(keep, z[b + e], __uint_as_float(v[e]));
      }
      fence_before();
      if (!STATES && c + 1 < chunks) {
        if (!(ok = __all_sync(0xFFFFFFFFu, wait_for(z_empty, c & 1, &failed)))) break;
        show();
      }
    }
    if (w.z_out && ok && r < w.dy && !(STATES && it.len == 0)) {
#pragma unroll
      for (int d = 0; d < D; ++d)
        if (d < w.du) w.z_out[at + d * w.dy + r] = z[d];
    }
  } else if (!STATES) {
    const int quad = warp % 4, i = quad * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const Val<2> near_by = fill<2>(w.w_near);
    for (int c = 0; c < chunks; ++c) {
      const int from = first_of(c), n = min(kTokens, it.len - from);
      if (!(ok = __all_sync(0xFFFFFFFFu, wait_for(p_full, c & 1, &failed)))) break;
      fence_after();
      // P' takes the place of columns of P that have been read
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        uint32_t packed[16] = {};
        if (late ? b * 32 + 31 >= quad * 32 : b * 32 <= quad * 32 + 31) {
          uint32_t v[32];
          tmem_ld32(lanes + P_AT + b * 32, v);
          tmem_wait_ld();
          const int away0 = late ? b * 32 - i : i - b * 32;
          const float step = late ? lg : -lg, start = away0 * lg;
          const int end = late ? n - b * 32 : 32;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            Val<2> p = mul_(Val<2>{{__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])}}, near_by);
            p = mul_(p, Val<2>{{exp2_fast(fmaf(2 * e, step, start)), exp2_fast(fmaf(2 * e + 1, step, start))}});
#pragma unroll
            for (int f = 0; f < 2; ++f) {
              const int j = 2 * e + f;
              if (late ? away0 + j < 0 || j >= end : away0 - j < 0) p.v[f] = 0.0f;
            }
            packed[e] = pack<T, 2>(p.v);
          }
        }
        tmem_st16(lanes + P_AT + b * 16, packed);
      }
      tmem_wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(p_ready);
      if (!(ok = __all_sync(0xFFFFFFFFu, wait_for(o_full, c & 1, &failed)))) break;
      fence_after();
      const bool there = i < n;
      const float by = there ? power[late ? n - 1 - i : i + 1] * w.w_row : 0.0f;
      T* out = static_cast<T*>(w.out) + (int64_t)(it.first + from + i) * w.out_ld + (int64_t)h * w.out_head;
#pragma unroll
      for (int b = 0; b < D; b += 32) {
        uint32_t x[32], y[32], packed[16];
        tmem_ld32(lanes + FAR + b, x);
        tmem_ld32(lanes + NEAR + b, y);
        tmem_wait_ld();
        if (b + 32 == D) {
          fence_before();
          __syncwarp();
          if (lane == 0) arrive(o_empty);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const Val<2> v = fma_(Val<2>{{__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])}}, fill<2>(by),
                                Val<2>{{__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])}});
          packed[e] = pack<T, 2>(v.v);
        }
        if (!there) continue;
        if (g.align[which] == 32 && b + 32 <= w.dy) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + b + 16 * e), DGC_I8(packed, 8 * e) : "memory");
        } else if (g.align[which] >= 16) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (b + 8 * e + 8 <= w.dy) {
              *reinterpret_cast<uint4*>(out + b + 8 * e) = make_uint4(packed[4 * e], packed[4 * e + 1], packed[4 * e + 2], packed[4 * e + 3]);
            } else {
#pragma unroll
              for (int f = 0; f < 8; ++f)
                if (b + 8 * e + f < w.dy)
                  store_word<T, 1>(out + b + 8 * e + f, f % 2 ? packed[4 * e + f / 2] >> 16 : packed[4 * e + f / 2] & 0xFFFFu);
            }
          }
        } else {
#pragma unroll
          for (int f = 0; f < 32; ++f)
            if (b + f < w.dy) store_word<T, 1>(out + b + f, f % 2 ? packed[f / 2] >> 16 : packed[f / 2] & 0xFFFFu);
        }
      }
    }
  }
  fence_before();
  __syncthreads();
  if (failed) let_copies_end();
  fence_after();
  if (warp == 1) tmem_free<1>(tmem, 512);
}

}  // namespace dgc
