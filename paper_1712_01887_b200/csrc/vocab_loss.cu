// Softmax cross entropy over a large vocabulary, from hidden rows and output matrix (sm_100a): kernels and
// C ABI.
//
//   l = h W^T + bias,   loss_r = log sum_j exp(l_rj) - l_{r, y_r}
//   G_r = dloss_r (softmax(l_r) - onehot(y_r)),   dh = G W,   dweight = G^T h,   dbias = sum_r G_r
//
// The logits exist a tile at a time.  Forward, a tile leaves each of its rows' largest logit and the sum
// of exponentials under it; one small kernel joins these.  Backward forms the tiles again, a piece of the
// vocabulary after the other: the piece of G goes to a workspace in the call's type, and two
// products take it from there.
//
// Padding rows (a label outside the vocabulary) are taken as rows of zeros: whatever they hold, nothing of
// it enters a product (0 times a NaN would).
//
// In DGC_F16, G is kept times a power of two that brings the largest |dloss| to 2^10 .. 2^11: a mean's
// dloss (1 over the rows) times a small probability would be below the type's range.

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "attention.cuh"
#include "tensor.cuh"

using namespace dgc;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kPieceBytes = 128 << 20;   // of G in the workspace
constexpr int kSms = 148;

// ------------------------------------------------------------------ the products
// Four products, C [m][n] = sum_k A(m, k) B(n, k):
//   kStats, kGrad   A = h,  B = W        rows of K in both
//   kDh             A = G,  B = W^T      (B: rows of N)
//   kDw             A = G^T, B = h^T     (rows of M, rows of N)
// A pair of blocks makes a tile of 256 x kN<T>: each holds the sums of its 128 rows in its tensor memory,
// loads its half of A's and of B's rows, and the first block's thread issues the products of both.  The
// tensor memory holds two tiles, so that one is taken out while the next is formed.
//
// 32-bit matrices are three bf16 planes (8 bits of the significand each; the planes' sum is the number), and
// of the nine products of planes the six that reach 2^-24 are formed.  The sums leave the tensor memory
// every kInterval steps of K and are added up in registers: a tensor core cuts off where an addition would round, and over
// a long K that would show (a relative 2^-24 a step, all to one side).
enum { kStats = 0, kGrad = 1, kDh = 2, kDw = 3 };
template <class T> constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
template <class T> constexpr int kPairs = sizeof(T) == 4 ? 6 : 1;
template <class T> constexpr int kN = sizeof(T) == 4 ? 128 : 256;
template <class T> constexpr int kInterval = sizeof(T) == 4 ? 2 : 1 << 30;
template <class T> using Operand = std::conditional_t<std::is_same_v<T, __half>, __half, __nv_bfloat16>;
constexpr int kM = 256, kK = 64, kThreads = 384, kRing = 196608, kStaging = 8 * 4096;
constexpr int kSharedBytes = 1024 + kRing + kStaging;

struct ProductArgs {
  CUtensorMap a, b, g;                // g: G, to be written (kGrad)
  int32_t m, n, k_blocks, tiles_m, tiles_n, splits, m_first;   // m_first: neighbours in M follow one another
  int32_t n0, vocab;                  // n0: the vocabulary's place of column 0
  const void* bias;
  const int32_t* labels;
  float2* parts;                      // kStats: [half tiles of n][m]
  float* picked;                      // kStats: the label's logit
  const float* stats;                 // kGrad: maximum and sum of each row
  const float* dloss;
  const float* scale;                 // G's factor
  float* sum;                         // kDh: [splits][m][ldc]
  void* c;                            // kDw
  int64_t ldc;
  int32_t add, wide;                  // kDh: sum holds something; kDw: rows of c are 16-byte aligned
};

template <class T>
__device__ __forceinline__ void work_item(const ProductArgs& g, int item, int& m0, int& n0, int& k0, int& k1, int& split) {
  const int tiles = g.tiles_m * g.tiles_n, t = item % tiles;
  split = item / tiles;
  const int tm = g.m_first ? t % g.tiles_m : t / g.tiles_n, tn = g.m_first ? t / g.tiles_m : t % g.tiles_n;
  m0 = tm * kM;
  n0 = tn * kN<T>;
  k0 = (int)((int64_t)g.k_blocks * split / g.splits);
  k1 = (int)((int64_t)g.k_blocks * (split + 1) / g.splits);
}

// Which planes the p-th product of a step multiplies.
__device__ __forceinline__ int plane_a(int p) { return p < 2 ? 0 : p < 4 ? 1 : p == 4 ? 0 : 2; }
__device__ __forceinline__ int plane_b(int p) { return p == 4 ? 2 : p == 5 ? 0 : p & 1; }

// The three planes of a 32-bit number: each remainder is exact.
__device__ __forceinline__ void planes_of(float v, __nv_bfloat16 (&p)[3]) {
  p[0] = __float2bfloat16_rn(v);
  float r = v - __bfloat162float(p[0]);
  if (!(fabsf(v) < INFINITY)) r = 0.0f;   // an infinity or a NaN is the first plane's alone
  p[1] = __float2bfloat16_rn(r);
  r -= __bfloat162float(p[1]);
  p[2] = __float2bfloat16_rn(r);
}

// 32 columns of 16-bit numbers of a lane's row, into half `half` of a 32 x 64 tile in the 128-byte swizzle.
template <class O>
__device__ __forceinline__ void stage_row(uint32_t tile, int row, int half, const uint32_t (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t at = tile + row * 128 + (((half * 4 + j) ^ (row & 7)) << 4);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[4 * j]), "r"(w[4 * j + 1]), "r"(w[4 * j + 2]), "r"(w[4 * j + 3]) : "memory");
  }
}

template <class T, int MODE>
__global__ void __launch_bounds__(kThreads, 1) k_product(const __grid_constant__ ProductArgs g) {
  using O = Operand<T>;
  constexpr bool A_TURNED = MODE == kDw, B_TURNED = MODE >= kDh;
  constexpr int N = kN<T>, HALF = N / 2, B_ROWS = N / 2, A_BYTES = 128 * 128, B_BYTES = B_ROWS * 128, STAGE = A_BYTES + B_BYTES;
  constexpr int STAGES = kRing / STAGE, COLUMNS = 2 * N;
  extern __shared__ char dynamic[];
  __shared__ __align__(8) uint64_t bars[2 * 8 + 4];
  __shared__ uint32_t tmem_at;
  __shared__ volatile int failed;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = blockIdx.x & 1;
  const uint32_t ring = (shared_u32(dynamic) + 1023) & ~1023u, staging = ring + kRing;
  const auto full = [&](int s) { return shared_u32(bars + s); };
  const auto empty = [&](int s) { return shared_u32(bars + 8 + s); };
  const auto tile_full = [&](int b) { return shared_u32(bars + 16 + b); };
  const auto tile_empty = [&](int b) { return shared_u32(bars + 18 + b); };
  if (tid == 0) {
    failed = 0;
    for (int s = 0; s < STAGES; ++s) { barrier_init(full(s), 1); barrier_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { barrier_init(tile_full(b), 1); barrier_init(tile_empty(b), 16); }
    barrier_init_visible();
    prefetch_map(&g.a);
    prefetch_map(&g.b);
  }
  if (warp == 2) tmem_alloc<2>(shared_u32(&tmem_at), COLUMNS);
  fence_before();
  __syncthreads();
  cluster_barrier();
  fence_after();
  pdl_enter();
  const uint32_t tmem = tmem_at;
  const int items = g.tiles_m * g.tiles_n * g.splits, first = blockIdx.x / 2, step = gridDim.x / 2;
  int m0, n0, k0, k1, split;

  if (warp == 0) {
    if (elect_one()) {
      int stage = 0, round = 0;
      bool ok = true;
      for (int item = first; item < items && ok; item += step) {
        work_item<T>(g, item, m0, n0, k0, k1, split);
        for (int kp = k0 * kPairs<T>; kp < k1 * kPairs<T>; ++kp) {
          const int k = kp / kPairs<T> * kK, pair = kp % kPairs<T>;
          if (!(ok = wait_for(empty(stage), (round & 1) ^ 1, &failed))) break;
          const uint32_t bar = in_block(full(stage), 0), a = ring + stage * STAGE, b = a + A_BYTES;
          if (rank == 0) arrive_expect(full(stage), 2 * STAGE);
          const int pa = plane_a(pair), pb = plane_b(pair), ma = m0 + rank * 128, nb = n0 + rank * B_ROWS;
          if (A_TURNED) {
            load_tile<2>(a, &g.a, bar, ma, k, pa);
            load_tile<2>(a + A_BYTES / 2, &g.a, bar, ma + 64, k, pa);
          } else {
            load_tile<2>(a, &g.a, bar, k, ma, pa);
          }
          if (B_TURNED) {
#pragma unroll
            for (int i = 0; i < B_ROWS / 64; ++i) load_tile<2>(b + i * 8192, &g.b, bar, nb + 64 * i, k, pb);
          } else {
            load_tile<2>(b, &g.b, bar, k, nb, pb);
          }
          if (++stage == STAGES) { stage = 0; ++round; }
        }
      }
    }
  } else if (warp == 1 && rank == 0) {
    if (elect_one()) {
      constexpr uint32_t what = product_descriptor(kM, N, std::is_same_v<O, __nv_bfloat16>, A_TURNED, B_TURNED);
      int stage = 0, round = 0, tile = 0;
      bool ok = true;
      for (int item = first; item < items && ok; item += step) {
        work_item<T>(g, item, m0, n0, k0, k1, split);
        for (int kb = k0; kb < k1 && ok;) {
          const int end = k1 - kb < kInterval<T> ? k1 : kb + kInterval<T>, buffer = tile & 1;
          if (!(ok = wait_for(tile_empty(buffer), (tile / 2 & 1) ^ 1, &failed))) break;
          fence_after();
          bool add = false;
          for (int kp = kb * kPairs<T>; kp < end * kPairs<T>; ++kp) {
            if (!(ok = wait_for(full(stage), round & 1, &failed))) break;
            fence_after();
            const uint64_t a = tile_descriptor(ring + stage * STAGE, A_TURNED ? A_BYTES / 2 : 16);
            const uint64_t b = tile_descriptor(ring + stage * STAGE + A_BYTES, B_TURNED ? 8192 : 16);
#pragma unroll
            for (int i = 0; i < kK / 16; ++i) {
              product<2>(tmem + buffer * N, a + i * (A_TURNED ? 2048 : 32) / 16, b + i * (B_TURNED ? 2048 : 32) / 16, what, add);
              add = true;
            }
            commit<2>(empty(stage));
            if (++stage == STAGES) { stage = 0; ++round; }
          }
          if (!ok) break;
          commit<2>(tile_full(buffer));
          ++tile;
          kb = end;
        }
      }
    }
  } else if (warp >= 4) {
    const int quad = warp % 4, half = (warp - 4) / 4;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + half * HALF, mine = staging + (warp - 4) * 4096;
    uint32_t drained[2] = {in_block(tile_empty(0), 0), in_block(tile_empty(1), 0)};
    int tile = 0;
    bool ok = true;
    const float factor = MODE == kGrad || MODE == kDw ? *g.scale : 1.0f;
    for (int item = first; item < items && ok; item += step) {
      work_item<T>(g, item, m0, n0, k0, k1, split);
      const int row0 = m0 + rank * 128 + quad * 32, row = row0 + lane, col0 = n0 + half * HALF;
      const bool there = row < g.m;
      // what the row needs beside its sums
      float top = -FLT_MAX, sum = 0.0f, coef = 0.0f, weight = 0.0f;
      bool labelled = false;
      uint32_t y = 0xC0000000u;   // the label's column (a label in another piece has one outside this); of padding rows none
      if (MODE <= kGrad && there) {
        const int label = g.labels[row];
        labelled = label >= 0 && label < g.vocab;
        if (labelled) y = (uint32_t)(label - g.n0);
      }
      if (MODE == kGrad && labelled) {
        top = g.stats[2 * (int64_t)row];
        sum = g.stats[2 * (int64_t)row + 1];
        weight = g.dloss[row] * factor;
        coef = sum == 0.0f ? 0.0f : weight / sum;
      }
      float acc[sizeof(T) == 4 ? HALF : 1];
      if constexpr (sizeof(T) == 4) {
        for (int kb = k0; kb < k1 && ok; kb = k1 - kb < kInterval<T> ? k1 : kb + kInterval<T>, ++tile) {
          if (!(ok = __all_sync(0xFFFFFFFFu, wait_for(tile_full(tile & 1), tile / 2 & 1, &failed)))) break;
          fence_after();
#pragma unroll
          for (int c = 0; c < HALF / 32; ++c) {
            uint32_t w[32];
            tmem_ld32(lanes + (tile & 1) * N + c * 32, w);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[c * 32 + i] = kb == k0 ? __uint_as_float(w[i]) : acc[c * 32 + i] + __uint_as_float(w[i]);
          }
          fence_before();
          __syncwarp();
          if (lane == 0) arrive_remote(drained[tile & 1]);
        }
      } else {
        ok = __all_sync(0xFFFFFFFFu, wait_for(tile_full(tile & 1), tile / 2 & 1, &failed));
        fence_after();
      }
      if (!ok) break;
#pragma unroll
      for (int c = 0; c < HALF / 32; ++c) {
        float v[32];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = acc[c * 32 + i];
        } else {
          uint32_t w[32];
          tmem_ld32(lanes + (tile & 1) * N + c * 32, w);
          tmem_wait_ld();
          if (c == HALF / 32 - 1) {
            fence_before();
            __syncwarp();
            if (lane == 0) arrive_remote(drained[tile & 1]);
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(w[i]);
        }
        const int col = col0 + c * 32;
        if (MODE <= kGrad) {
          if (g.bias && col < g.n) {
            const T* bias = static_cast<const T*>(g.bias) + g.n0 + col;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (col + i < g.n) v[i] += to_float<T>(bias[i]);
          }
          if (col + 32 > g.n) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (col + i >= g.n) v[i] = -INFINITY;
          }
        }
        if (MODE == kStats) {
          float best = v[0];
#pragma unroll
          for (int i = 1; i < 32; ++i) best = fmaxf(best, v[i]);
          if (best > top) {
            sum *= exp2_fast((top - best) * kLog2e);
            top = best;
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) sum += exp2_fast((v[i] - top) * kLog2e);
          if (y - (uint32_t)col < 32u) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (y - (uint32_t)col == (uint32_t)i) g.picked[row] = v[i];
          }
        } else if (MODE == kGrad) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = exp2_fast((v[i] - top) * kLog2e) * coef;
          if (y - (uint32_t)col < 32u) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (y - (uint32_t)col == (uint32_t)i) v[i] -= weight;
          }
          if (!(weight != 0.0f)) {   // a padding row, whatever the sums are: zeros
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.0f;
          }
          if constexpr (sizeof(T) == 4) {
            // a plane a tile: three tiles of 32 x 32 would fit the staging, but not the swizzle's rows of 64
#pragma unroll 1
            for (int p = 0; p < 3; ++p) {
              uint32_t w[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float lo = __bfloat162float(__float2bfloat16_rn(v[2 * i])), hi = __bfloat162float(__float2bfloat16_rn(v[2 * i + 1]));
                const float two[2] = {lo, hi};
                w[i] = pack<O, 2>(two);
                v[2 * i] -= lo;
                v[2 * i + 1] -= hi;
              }
              char* to = static_cast<char*>(g.c) + ((int64_t)p * g.m + row) * g.ldc * 2 + (int64_t)col * 2;
              if (there) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (col + 8 * j < g.ldc) *reinterpret_cast<uint4*>(to + 16 * j) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
              }
            }
          } else {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float two[2] = {v[2 * i], v[2 * i + 1]};
              w[i] = pack<O, 2>(two);
            }
            if (c % 2 == 0) {
              if (lane == 0) store_wait_read();
              __syncwarp();
            }
            stage_row<O>(mine, lane, c % 2, w);
            if (c % 2 == 1) {
              shared_to_async();
              __syncwarp();
              if (lane == 0 && col0 + (c - 1) * 32 < g.n && row0 < g.m) {
                store_tile(&g.g, mine, col0 + (c - 1) * 32, row0, 0);
                store_commit();
              }
            }
          }
        } else if (MODE == kDh) {
          if (there) {
            float* to = g.sum + ((int64_t)split * g.m + row) * g.ldc + col;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              if (col + 4 * j >= g.ldc) continue;
              float4 x = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
              if (g.add) {
                const float4 o = *reinterpret_cast<const float4*>(to + 4 * j);
                x.x += o.x; x.y += o.y; x.z += o.z; x.w += o.w;
              }
              *reinterpret_cast<float4*>(to + 4 * j) = x;
            }
          }
        } else {
          if (there) {
            T* to = static_cast<T*>(g.c) + (int64_t)row * g.ldc + col;
            const float inverse = 1.0f / factor;
            if (g.wide && col + 32 <= g.n) {
              constexpr int E = 16 / sizeof(T);
#pragma unroll
              for (int j = 0; j < 32 / E; ++j) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if constexpr (sizeof(T) == 4) {
                    w[i] = __float_as_uint(v[4 * j + i] * inverse);
                  } else {
                    const float two[2] = {v[8 * j + 2 * i] * inverse, v[8 * j + 2 * i + 1] * inverse};
                    w[i] = pack<T, 2>(two);
                  }
                }
                *reinterpret_cast<uint4*>(to + j * E) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (col + i < g.n) to[i] = from_float<T>(v[i] * inverse);
            }
          }
        }
      }
      if (MODE == kStats && there && col0 < g.n)
        g.parts[(int64_t)(col0 / HALF) * g.m + row] = make_float2(top, sum);
      if constexpr (sizeof(T) != 4) ++tile;
    }
    if (MODE == kGrad && sizeof(T) != 4 && lane == 0) store_wait_all();
  }
  fence_before();
  __syncthreads();
  if (failed) let_copies_end();
  cluster_barrier();   // (the other block may still load, multiply and arrive here)
  fence_after();
  if (warp == 2) tmem_free<2>(tmem, COLUMNS);
}

// ------------------------------------------------------------------ around the products
// The halves' maxima and sums become the row's, and its loss.  32 rows a block, 16 threads a row.
__global__ void __launch_bounds__(512) k_row_loss(const float2* parts, int halves, const float* picked, const int32_t* labels, int32_t rows,
                                                  int32_t vocab, float* loss, float* stats) {
  pdl_enter();
  __shared__ float2 held[16][33];
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32, r = blockIdx.x * 32 + lane;
  float top = -FLT_MAX, sum = 0.0f;
  if (r < rows) {
    for (int t0 = w; t0 < halves; t0 += 16 * 8) {   // (eight loads under way at once)
      float2 p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = t0 + 16 * i < halves ? parts[(int64_t)(t0 + 16 * i) * rows + r] : make_float2(-FLT_MAX, 0.0f);
      float best = top;
#pragma unroll
      for (int i = 0; i < 8; ++i) best = fmaxf(best, p[i].x);
      sum *= exp2f((top - best) * kLog2e);
      top = best;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += p[i].y * exp2f((p[i].x - top) * kLog2e);
    }
  }
  held[w][lane] = make_float2(top, sum);
  __syncthreads();
  if (w || r >= rows) return;
  for (int i = 1; i < 16; ++i) top = fmaxf(top, held[i][lane].x);
  sum = 0.0f;
  for (int i = 0; i < 16; ++i) sum += held[i][lane].y * exp2f((held[i][lane].x - top) * kLog2e);
  const int y = labels[r];
  if (loss) {
    float l = 0.0f;
    if (y >= 0 && y < vocab) {
      const float own = picked[r];
      l = own == -INFINITY ? INFINITY : logf(sum) + (top - own);
    }
    loss[r] = l;
  }
  if (stats) { stats[2 * (int64_t)r] = top; stats[2 * (int64_t)r + 1] = sum; }
}

// A matrix as the products take it: rows on 16 bytes, 32-bit numbers in planes, padding rows (`labels` given)
// zeros.  A thread makes 8 elements.
template <class T>
__global__ void __launch_bounds__(256) k_pack(const T* from, int64_t ld, const int32_t* labels, int32_t vocab, int64_t rows, int32_t width,
                                              int32_t to_ld, Operand<T>* to) {
  pdl_enter();
  const int groups = to_ld / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, r = i / groups;
  if (r >= rows) return;
  const int c = (int)(i - r * groups) * 8;
  bool there = true;
  if (labels) {
    const int y = labels[r];
    there = y >= 0 && y < vocab;
  }
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = there && c + e < width ? to_float<T>(from[r * ld + c + e]) : 0.0f;
#pragma unroll
  for (int p = 0; p < kPlanes<T>; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) {
        __nv_bfloat16 a[3], b[3];
        planes_of(v[2 * e], a);
        planes_of(v[2 * e + 1], b);
        const float two[2] = {__bfloat162float(a[p]), __bfloat162float(b[p])};
        w[e] = pack<Operand<T>, 2>(two);
      } else {
        const float two[2] = {v[2 * e], v[2 * e + 1]};
        w[e] = pack<Operand<T>, 2>(two);
      }
    }
    *reinterpret_cast<uint4*>(to + (p * rows + r) * to_ld + c) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// G's factor: 1, or the power of two stated above.
__global__ void __launch_bounds__(1024) k_scale(const float* dloss, const int32_t* labels, int32_t vocab, int64_t rows, int narrow, float* scale) {
  pdl_enter();
  __shared__ float best[32];
  float top = 0.0f;
  if (narrow)
    for (int64_t r = threadIdx.x; r < rows; r += 1024)
      if (labels[r] >= 0 && labels[r] < vocab) top = fmaxf(top, fabsf(dloss[r]));
#pragma unroll
  for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  if (threadIdx.x % 32 == 0) best[threadIdx.x / 32] = top;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < 32; ++i) top = fmaxf(top, best[i]);
  *scale = narrow && top > 0x1p-100f && top < 0x1p100f ? exp2f(10.0f - floorf(log2f(top))) : 1.0f;
}

// dbias: the columns' sums of G.  A thread adds two columns of every 32nd row, eight loads under way at once.
template <class T>
__global__ void __launch_bounds__(1024) k_bias_grad(const Operand<T>* g, int64_t ld, int64_t rows, int32_t n, const float* scale, T* out) {
  pdl_enter();
  using O = Operand<T>;
  __shared__ float part[32][64];
  const int lane = threadIdx.x % 32, c = blockIdx.x * 64 + lane * 2, w = threadIdx.x / 32;
  const int64_t end = rows * kPlanes<T>;
  float s[2] = {};
  if (c < n)
    for (int64_t r0 = w; r0 < end; r0 += 32 * 8) {
      uint32_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = r0 + 32 * i < end ? *reinterpret_cast<const uint32_t*>(g + (r0 + 32 * i) * ld + c) : 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float two[2];
        unpack<O, 2>(v[i], two);
        s[0] += two[0];
        s[1] += two[1];
      }
    }
  part[w][lane * 2] = s[0];
  part[w][lane * 2 + 1] = s[1];
  __syncthreads();
  const int col = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x >= 64 || col >= n) return;
  float all = 0.0f;
  for (int i = 0; i < 32; ++i) all += part[i][threadIdx.x];
  out[col] = from_float<T>(all / *scale);
}

// dh from the splits' sums.
template <class T>
__global__ void __launch_bounds__(256) k_finish(const float* sum, int64_t ld, int splits, int64_t rows, int32_t width, const float* scale, T* out, int64_t out_ld) {
  pdl_enter();
  const int64_t r = blockIdx.x;
  const float inverse = 1.0f / *scale;
  for (int c = threadIdx.x; c < width; c += 256) {
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += sum[(s * rows + r) * ld + c];
    out[r * out_ld + c] = from_float<T>(v * inverse);
  }
}

// ------------------------------------------------------------------ host
struct Plan {
  int32_t planes, tile_n, splits, ld;      // ld: of packed rows
  int64_t piece, halves;
  int64_t kept, picked, rows, weight, parts, g, sum, bytes;   // offsets in the workspace
  bool packed;                             // the output matrix
};
Plan plan_of(const dgc_vocab_loss* d, bool gradient) {
  Plan p{};
  const int64_t R = std::max<int64_t>(d->rows, 1), V = d->vocab;
  const auto take = [&](int64_t bytes) { const int64_t at = p.bytes; p.bytes += (bytes + 255) / 256 * 256; return at; };
  const bool f32 = d->dtype == DGC_F32;
  p.planes = f32 ? 3 : 1;
  p.tile_n = f32 ? kN<float> : kN<__half>;
  p.ld = (d->hidden + 7) / 8 * 8;
  p.halves = (V + p.tile_n / 2 - 1) / (p.tile_n / 2);
  p.packed = f32 || misaligned(d->weight.data, 16) || d->weight.ld % 8 != 0;
  take(256);   // the factor
  p.kept = take(R * 8);
  p.picked = take(R * 4);
  p.rows = take(R * p.ld * 2 * p.planes);
  p.weight = p.packed ? take(V * p.ld * 2 * p.planes) : 0;
  const int64_t most = std::max<int64_t>(kPieceBytes / (R * 2 * p.planes) / 256 * 256, 256), pieces = (V + most - 1) / most;
  p.piece = ((V + pieces - 1) / pieces + 255) / 256 * 256;
  p.parts = p.g = take(std::max<int64_t>(R * p.halves * 8, gradient ? R * p.piece * 2 * p.planes : 0));   // (the sums are used up before G comes)
  // dh has few tiles and a long K: as many parts of K as there are blocks for
  const int64_t tiles = (R + kM - 1) / kM * ((d->hidden + p.tile_n - 1) / p.tile_n), k_blocks = (std::min(p.piece, V) + kK - 1) / kK;
  p.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kSms / 2 / tiles, k_blocks / 8));
  p.sum = gradient ? take(p.splits * R * p.ld * 4) : 0;
  return p;
}
inline bool bad_sizes(const dgc_vocab_loss* d) {
  return !d || bad_dtype(d->dtype) || d->vocab < 1 || d->vocab > INT32_MAX - 1023 || d->hidden < 1 || d->hidden > 65536 ||
         d->rows < 0 || d->rows > INT32_MAX - 1023;
}

template <class T, int MODE>
int32_t enqueue(ProductArgs& g, cudaStream_t s) {
  g.tiles_m = (g.m + kM - 1) / kM;
  g.tiles_n = (g.n + kN<T> - 1) / kN<T>;
  g.m_first = g.tiles_m < g.tiles_n;
  const int64_t items = (int64_t)g.tiles_m * g.tiles_n * g.splits;
  if (items > INT32_MAX / 2) return DGC_EINVAL;
  const int32_t rc = allow_shared<&k_product<T, MODE>>(kSharedBytes);
  if (rc != DGC_OK) return rc;
  launch_cluster(k_product<T, MODE>, dim3((unsigned)std::min<int64_t>(2 * items, kSms)), dim3(kThreads), kSharedBytes, s, 2u, g);
  return check_launch();
}

template <class T>
int32_t run(const dgc_vocab_loss* d, bool forward, bool gradient, cudaStream_t s) {
  using O = Operand<T>;
  constexpr bool BF16 = std::is_same_v<O, __nv_bfloat16>;
  constexpr int P = kPlanes<T>, HB = kN<T> / 2;
  const Plan p = plan_of(d, gradient);
  char* const work = static_cast<char*>(d->workspace);
  float* const scale = reinterpret_cast<float*>(work);
  float* const kept = reinterpret_cast<float*>(work + p.kept);
  float* const picked = reinterpret_cast<float*>(work + p.picked);
  float* const sum = reinterpret_cast<float*>(work + p.sum);
  O* const rows = reinterpret_cast<O*>(work + p.rows);
  O* const G = reinterpret_cast<O*>(work + p.g);
  const int32_t R = (int32_t)d->rows, V = d->vocab, D = d->hidden;
  const O* W = static_cast<const O*>(d->weight.data);
  int64_t w_ld = d->weight.ld;
  int32_t rc;
  const auto pack_rows = [&](const void* from, int64_t ld, const int32_t* labels, int64_t n, O* to) {
    const int64_t blocks = (n * (p.ld / 8) + 255) / 256;
    if (blocks > INT32_MAX) return DGC_EINVAL;
    launch(k_pack<T>, (unsigned)blocks, 256, 0, s, static_cast<const T*>(from), ld, labels, V, n, D, p.ld, to);
    return check_launch();
  };
  if ((rc = pack_rows(d->h.data, d->h.ld, d->labels, R, rows)) != DGC_OK) return rc;
  if (p.packed) {
    O* const to = reinterpret_cast<O*>(work + p.weight);
    if ((rc = pack_rows(d->weight.data, d->weight.ld, nullptr, V, to)) != DGC_OK) return rc;
    W = to;
    w_ld = p.ld;
  }
  ProductArgs g{};
  g.splits = 1; g.vocab = V; g.bias = d->bias; g.labels = d->labels; g.m = R; g.n = V; g.k_blocks = (D + kK - 1) / kK; g.scale = scale;
  if ((rc = tensor_map(&g.a, rows, BF16, D, R, P, p.ld, (int64_t)R * p.ld, 128)) != DGC_OK) return rc;
  if (forward) {
    if ((rc = tensor_map(&g.b, W, BF16, D, V, P, w_ld, (int64_t)V * w_ld, HB)) != DGC_OK) return rc;
    g.parts = reinterpret_cast<float2*>(work + p.parts);
    g.picked = picked;
    if ((rc = enqueue<T, kStats>(g, s)) != DGC_OK) return rc;
    launch(k_row_loss, (unsigned)((d->rows + 31) / 32), 512, 0, s, g.parts, (int)p.halves, picked, d->labels, R, V, d->loss,
           gradient ? kept : d->stats);
    if ((rc = check_launch()) != DGC_OK) return rc;
  }
  if (!gradient) return DGC_OK;
  launch(k_scale, 1, 1024, 0, s, d->dloss, d->labels, V, d->rows, std::is_same_v<T, __half> ? 1 : 0, scale);
  if ((rc = check_launch()) != DGC_OK) return rc;
  g.stats = forward ? kept : d->stats;
  g.dloss = d->dloss;
  for (int64_t v = 0; v < V; v += p.piece) {
    const int32_t n = (int32_t)std::min<int64_t>(p.piece, V - v);
    const O* const Wv = W + v * w_ld;
    g.n = n; g.n0 = (int32_t)v; g.c = G; g.ldc = p.piece;
    if ((rc = tensor_map(&g.b, Wv, BF16, D, n, P, w_ld, (int64_t)V * w_ld, HB)) != DGC_OK) return rc;
    if ((rc = tensor_map(&g.g, G, BF16, n, R, P, p.piece, (int64_t)R * p.piece, 32)) != DGC_OK) return rc;
    if ((rc = enqueue<T, kGrad>(g, s)) != DGC_OK) return rc;
    ProductArgs w{};     // dweight = G^T h
    w.m = n; w.n = D; w.k_blocks = (R + kK - 1) / kK; w.splits = 1; w.scale = scale;
    w.c = static_cast<T*>(d->dweight.data) + v * d->dweight.ld; w.ldc = d->dweight.ld;
    w.wide = !misaligned(w.c, 16) && w.ldc % (16 / (int)sizeof(T)) == 0;
    if ((rc = tensor_map(&w.a, G, BF16, n, R, P, p.piece, (int64_t)R * p.piece, kK)) != DGC_OK) return rc;
    if ((rc = tensor_map(&w.b, rows, BF16, D, R, P, p.ld, (int64_t)R * p.ld, kK)) != DGC_OK) return rc;
    if ((rc = enqueue<T, kDw>(w, s)) != DGC_OK) return rc;
    if (d->dbias) {
      launch(k_bias_grad<T>, (n + 63) / 64, 1024, 0, s, static_cast<const O*>(G), p.piece, d->rows, n, static_cast<const float*>(scale),
             static_cast<T*>(d->dbias) + v);
      if ((rc = check_launch()) != DGC_OK) return rc;
    }
    ProductArgs x{};     // dh = G W
    x.m = R; x.n = D; x.k_blocks = (n + kK - 1) / kK; x.splits = std::min(p.splits, x.k_blocks); x.scale = scale; x.sum = sum; x.ldc = p.ld; x.add = v != 0;
    if ((rc = tensor_map(&x.a, G, BF16, n, R, P, p.piece, (int64_t)R * p.piece, 128)) != DGC_OK) return rc;
    if ((rc = tensor_map(&x.b, Wv, BF16, D, n, P, w_ld, (int64_t)V * w_ld, kK)) != DGC_OK) return rc;
    if ((rc = enqueue<T, kDh>(x, s)) != DGC_OK) return rc;
  }
  launch(k_finish<T>, R, 256, 0, s, static_cast<const float*>(sum), (int64_t)p.ld, p.splits, d->rows, D, static_cast<const float*>(scale),
         static_cast<T*>(d->dh.data), d->dh.ld);
  return check_launch();
}

int32_t vocab_loss(const dgc_vocab_loss* d, bool forward, bool gradient, void* stream) {
  if (bad_sizes(d)) return DGC_EINVAL;
  const size_t es = element_size(d->dtype);
  if (bad_matrix(d->h, d->rows, d->hidden, es) || bad_matrix(d->weight, d->vocab, d->hidden, es) || misaligned(d->bias, es) ||
      misaligned(d->labels, 4) || misaligned(d->loss, 4) || misaligned(d->stats, 4) || misaligned(d->dloss, 4) ||
      misaligned(d->workspace, 256) || d->workspace_bytes < 0)
    return DGC_EINVAL;
  if (gradient && (bad_matrix(d->dh, d->rows, d->hidden, es) || bad_matrix(d->dweight, d->vocab, d->hidden, es) || misaligned(d->dbias, es)))
    return DGC_EINVAL;
  if (d->rows == 0 && !gradient) return DGC_OK;
  if (d->rows > 0 && (!d->labels || (forward && !d->loss) || (gradient && !d->dloss) || (gradient && !forward && !d->stats))) return DGC_EINVAL;
  if (!d->workspace || d->workspace_bytes < plan_of(d, gradient).bytes) return DGC_ECAPACITY;
  cudaStream_t s = as_stream(stream);
  if (d->rows == 0) {   // nothing was seen: gradients of zero
    DGC_CUDA(cudaMemset2DAsync(d->dweight.data, d->dweight.ld * es, 0, d->hidden * es, d->vocab, s));
    if (d->dbias) DGC_CUDA(cudaMemsetAsync(d->dbias, 0, d->vocab * es, s));
    return DGC_OK;
  }
  if (d->dtype == DGC_F32) return run<float>(d, forward, gradient, s);
  if (d->dtype == DGC_BF16) return run<__nv_bfloat16>(d, forward, gradient, s);
  return run<__half>(d, forward, gradient, s);
}

}  // namespace

extern "C" {

int64_t dgc_vocab_loss_workspace_bytes(const dgc_vocab_loss* d, int32_t gradient) {
  return bad_sizes(d) ? DGC_EINVAL : plan_of(d, gradient != 0).bytes;
}
int32_t dgc_tensor_check(void* stream) {
  DGC_CUDA(cudaStreamSynchronize(as_stream(stream)));
  int here = 0, there = 0;
  int32_t rc = take_waits_out(&here);
  if (rc == DGC_OK) rc = attention_waits_out(&there);
  return rc != DGC_OK ? rc : here || there ? DGC_ECUDA : DGC_OK;
}
int32_t dgc_vocab_loss_forward(const dgc_vocab_loss* d, void* stream) { return vocab_loss(d, true, false, stream); }
int32_t dgc_vocab_loss_backward(const dgc_vocab_loss* d, void* stream) { return vocab_loss(d, false, true, stream); }
int32_t dgc_vocab_loss_grad(const dgc_vocab_loss* d, void* stream) { return vocab_loss(d, true, true, stream); }

}  // extern "C"
