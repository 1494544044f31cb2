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

#include "common.cuh"

using namespace dgc;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 64, kDepth = 16;
constexpr int64_t kPieceBytes = 128 << 20;   // of G in the workspace
enum { kStats = 0, kGrad = 1, kOut = 2 };

struct ProductArgs {
  const void *a, *b;                  // element (m, k) at a[m am + k ak], (n, k) at b[n bn + k bk]
  int64_t am, ak, bn, bk;
  int32_t m, n, k, n0, vocab;         // n0: the vocabulary's place of column 0
  const void* bias;
  const int32_t* labels;
  float2* parts;                      // kStats: [m][tiles of n]
  float* picked;                      // kStats: the label's logit
  const float* stats;                 // kGrad: maximum and sum of each row
  const float* dloss;
  const float* scale;                 // kGrad: G's factor; kOut: its inverse behind it
  void* c;                            // kGrad: G [m][ldc]; kOut: the result
  float* sum;                         // kOut: [m][n], what came before; NULL: nothing
  int64_t ldc;
  int32_t first, last;                // kOut: of the pieces that are summed
};

template <class T, int MODE>
__global__ void __launch_bounds__(256) k_product(const ProductArgs g) {
  pdl_enter();
  __shared__ float A[kDepth][kTile + 4], Bm[kDepth][kTile + 4];
  __shared__ float C[MODE == kStats ? kTile : 1][kTile + 1];
  const int m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile, tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
  float acc[4][4] = {};
  const T* a = static_cast<const T*>(g.a);
  const T* b = static_cast<const T*>(g.b);
  for (int k0 = 0; k0 < g.k; k0 += kDepth) {
    __syncthreads();
    for (int e = tid; e < kTile * kDepth; e += 256) {
      const int ra = g.ak == 1 ? e / kDepth : e % kTile, ka = g.ak == 1 ? e % kDepth : e / kTile;
      A[ka][ra] = m0 + ra < g.m && k0 + ka < g.k ? to_float<T>(a[(m0 + ra) * g.am + (k0 + ka) * g.ak]) : 0.0f;
      const int rb = g.bk == 1 ? e / kDepth : e % kTile, kb = g.bk == 1 ? e % kDepth : e / kTile;
      Bm[kb][rb] = n0 + rb < g.n && k0 + kb < g.k ? to_float<T>(b[(n0 + rb) * g.bn + (k0 + kb) * g.bk]) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&A[k][ty * 4]), y = *reinterpret_cast<const float4*>(&Bm[k][tx * 4]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[i], ys[j], acc[i][j]);
    }
  }
  if (MODE == kOut) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
        if (m >= g.m || n >= g.n) continue;
        float v = acc[i][j];
        if (g.sum) {
          if (!g.first) v += g.sum[(int64_t)m * g.n + n];
          if (!g.last) { g.sum[(int64_t)m * g.n + n] = v; continue; }
        }
        static_cast<T*>(g.c)[m * g.ldc + n] = from_float<T>(v * (1.0f / *g.scale));
      }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j, word = g.n0 + n;
      float v = acc[i][j];
      if (g.bias && n < g.n) v += to_float<T>(static_cast<const T*>(g.bias)[word]);
      if (n >= g.n) v = -INFINITY;
      if (MODE == kStats) {
        C[ty * 4 + i][tx * 4 + j] = v;
        if (m < g.m && n < g.n && g.labels[m] == word) g.picked[m] = v;
      } else if (m < g.m && n < g.ldc) {
        const int y = g.labels[m];
        const float2 st = make_float2(g.stats[2 * (int64_t)m], g.stats[2 * (int64_t)m + 1]);
        float p = 0.0f;
        if (y >= 0 && y < g.vocab && n < g.n) {
          p = st.y == 0.0f ? 0.0f : exp2f((v - st.x) * kLog2e) / st.y;
          p = (p - (word == y ? 1.0f : 0.0f)) * g.dloss[m] * *g.scale;
        }
        static_cast<T*>(g.c)[m * g.ldc + n] = from_float<T>(p);
      }
    }
  if (MODE == kStats) {
    __syncthreads();
    if (tid < kTile && m0 + tid < g.m) {
      float top = -FLT_MAX, sum = 0.0f;
      for (int j = 0; j < kTile; ++j) top = fmaxf(top, C[tid][j]);
      for (int j = 0; j < kTile; ++j) sum += exp2f((C[tid][j] - top) * kLog2e);
      g.parts[(int64_t)(m0 + tid) * gridDim.x + blockIdx.x] = make_float2(top, sum);
    }
  }
}

// One warp a row: the tiles' maxima and sums become the row's, and its loss.
__global__ void __launch_bounds__(256) k_row_loss(const float2* parts, int tiles, const float* picked, const int32_t* labels,
                                                  int64_t rows, int32_t vocab, float* loss, float* stats) {
  pdl_enter();
  const int64_t r = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (r >= rows) return;
  float top = -FLT_MAX, sum = 0.0f;
  for (int t = lane; t < tiles; t += 32) top = fmaxf(top, parts[r * tiles + t].x);
#pragma unroll
  for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  for (int t = lane; t < tiles; t += 32) {
    const float2 p = parts[r * tiles + t];
    sum += p.y * exp2f((p.x - top) * kLog2e);
  }
#pragma unroll
  for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  if (lane) return;
  const int y = labels[r];
  if (loss) loss[r] = y >= 0 && y < vocab ? (picked[r] == -INFINITY ? INFINITY : logf(sum) + (top - picked[r])) : 0.0f;
  if (stats) { stats[2 * r] = top; stats[2 * r + 1] = sum; }
}

// The hidden rows as the products take them: padding rows are zeros.
template <class T>
__global__ void __launch_bounds__(256) k_take_rows(const T* h, int64_t ld, const int32_t* labels, int32_t vocab, int32_t hidden, T* to) {
  pdl_enter();
  const int64_t r = blockIdx.x;
  const int y = labels[r];
  const bool there = y >= 0 && y < vocab;
  for (int c = threadIdx.x; c < hidden; c += 256) to[r * hidden + c] = there ? h[r * ld + c] : from_float<T>(0.0f);
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

template <class T>
__global__ void __launch_bounds__(256) k_bias_grad(const T* g, int64_t ld, int64_t rows, int32_t n, const float* scale, T* out) {
  pdl_enter();
  __shared__ float part[8][32];
  const int c = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32;
  float s = 0.0f;
  if (c < n)
    for (int64_t r = w; r < rows; r += 8) s += to_float<T>(g[r * ld + c]);
  part[w][threadIdx.x % 32] = s;
  __syncthreads();
  if (w || c >= n) return;
  for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
  out[c] = from_float<T>(s / *scale);
}

// ------------------------------------------------------------------ host
struct Plan {
  int64_t piece, tiles, kept, parts, picked, rows, g, sum, bytes;   // offsets in the workspace
};
Plan plan_of(const dgc_vocab_loss* d, bool gradient) {
  Plan p{};
  const int64_t es = element_size(d->dtype), R = d->rows;
  const auto take = [&](int64_t bytes) { const int64_t at = p.bytes; p.bytes += (bytes + 255) / 256 * 256; return at; };
  p.tiles = (d->vocab + kTile - 1) / kTile;
  take(256);   // the factor
  p.kept = take(R * 8);
  p.picked = take(R * 4);
  p.rows = take(R * d->hidden * es);
  p.piece = std::min<int64_t>(std::max<int64_t>(kPieceBytes / (std::max<int64_t>(R, 1) * es) / 256 * 256, 256), (d->vocab + 7) / 8 * 8);
  p.parts = p.g = p.bytes;
  const int64_t parts = R * p.tiles * 8, g = gradient ? R * p.piece * es : 0;
  take(std::max(parts, g));   // the tiles' sums are used up before G comes
  p.sum = gradient ? take(R * d->hidden * 4) : 0;
  return p;
}
inline bool bad_sizes(const dgc_vocab_loss* d) {
  return !d || bad_dtype(d->dtype) || d->vocab < 1 || d->vocab > INT32_MAX - 1023 || d->hidden < 1 || d->hidden > 65536 ||
         d->rows < 0 || d->rows > INT32_MAX - 1023;
}

template <class T, int MODE>
int32_t product(const ProductArgs& g, int64_t columns, cudaStream_t s) {
  launch(k_product<T, MODE>, dim3((unsigned)((columns + kTile - 1) / kTile), (g.m + kTile - 1) / kTile), 256, 0, s, g);
  return check_launch();
}

template <class T>
int32_t run(const dgc_vocab_loss* d, bool forward, bool gradient, cudaStream_t s) {
  const Plan p = plan_of(d, gradient);
  char* const work = static_cast<char*>(d->workspace);
  float* const scale = reinterpret_cast<float*>(work);
  float* const kept = reinterpret_cast<float*>(work + p.kept);
  float* const picked = reinterpret_cast<float*>(work + p.picked);
  float* const sum = reinterpret_cast<float*>(work + p.sum);
  T* const rows = reinterpret_cast<T*>(work + p.rows);
  T* const G = reinterpret_cast<T*>(work + p.g);
  const int32_t R = (int32_t)d->rows, V = d->vocab, D = d->hidden;
  int32_t rc;
  launch(k_take_rows<T>, R, 256, 0, s, static_cast<const T*>(d->h.data), d->h.ld, d->labels, V, D, rows);
  if ((rc = check_launch()) != DGC_OK) return rc;
  ProductArgs g{};
  g.a = rows; g.am = D; g.ak = 1; g.b = d->weight.data; g.bn = d->weight.ld; g.bk = 1;
  g.m = R; g.n = V; g.k = D; g.vocab = V; g.bias = d->bias; g.labels = d->labels;
  if (forward) {
    g.parts = reinterpret_cast<float2*>(work + p.parts);
    g.picked = picked;
    if ((rc = product<T, kStats>(g, V, s)) != DGC_OK) return rc;
    launch(k_row_loss, (unsigned)((d->rows + 7) / 8), 256, 0, s, g.parts, (int)p.tiles, picked, d->labels, d->rows, V, d->loss,
           gradient ? kept : d->stats);
    if ((rc = check_launch()) != DGC_OK) return rc;
  }
  if (!gradient) return DGC_OK;
  launch(k_scale, 1, 1024, 0, s, d->dloss, d->labels, V, d->rows, std::is_same_v<T, __half> ? 1 : 0, scale);
  if ((rc = check_launch()) != DGC_OK) return rc;
  g.stats = forward ? kept : d->stats;
  g.dloss = d->dloss; g.scale = scale;
  for (int64_t v = 0; v < V; v += p.piece) {
    const int32_t n = (int32_t)std::min<int64_t>(p.piece, V - v);
    ProductArgs a = g;
    a.b = static_cast<const T*>(d->weight.data) + v * d->weight.ld;
    a.n = n; a.n0 = (int32_t)v; a.c = G; a.ldc = p.piece;
    if ((rc = product<T, kGrad>(a, p.piece, s)) != DGC_OK) return rc;
    ProductArgs w{};     // dweight = G^T h
    w.a = G; w.am = 1; w.ak = p.piece; w.b = rows; w.bn = 1; w.bk = D; w.m = n; w.n = D; w.k = R; w.scale = scale;
    w.c = static_cast<T*>(d->dweight.data) + v * d->dweight.ld; w.ldc = d->dweight.ld;
    if ((rc = product<T, kOut>(w, D, s)) != DGC_OK) return rc;
    if (d->dbias) {
      launch(k_bias_grad<T>, (n + 31) / 32, 256, 0, s, static_cast<const T*>(G), p.piece, d->rows, n, static_cast<const float*>(scale),
             static_cast<T*>(d->dbias) + v);
      if ((rc = check_launch()) != DGC_OK) return rc;
    }
    ProductArgs x{};     // dh = G W
    x.a = G; x.am = p.piece; x.ak = 1; x.b = a.b; x.bn = 1; x.bk = d->weight.ld; x.m = R; x.n = D; x.k = n; x.scale = scale;
    x.c = d->dh.data; x.ldc = d->dh.ld; x.sum = sum; x.first = v == 0; x.last = v + n >= V;
    if ((rc = product<T, kOut>(x, D, s)) != DGC_OK) return rc;
  }
  return DGC_OK;
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
int32_t dgc_vocab_loss_forward(const dgc_vocab_loss* d, void* stream) { return vocab_loss(d, true, false, stream); }
int32_t dgc_vocab_loss_backward(const dgc_vocab_loss* d, void* stream) { return vocab_loss(d, false, true, stream); }
int32_t dgc_vocab_loss_grad(const dgc_vocab_loss* d, void* stream) { return vocab_loss(d, true, true, stream); }

}  // extern "C"
