// What the kernels of linear attention share: the walk that all of them are, and how a launch's blocks
// find their part of it.
//
//   forward            S_t = g S_{t-1} + k_t v_t^T,            o_t = c S_t^T q_t
//   gradients          dS_t = E_t + c q_t do_t^T,  E_{t-1} = g dS_t
//                      dq_t = c S_t do_t,   dk_t = dS_t v_t,   dv_t = dS_t^T k_t
//
// Each of the four is one walk  Z_t = g Z_{t-1} + w x_t y_t^T,  row_t = Z_t^T u_t  over a sequence, with other roles:
//   out  u = q,  x = k,  y = v    early (from the first token on), Z = S
//   dq   u = do, x = v,  y = k    early, Z = S^T
//   dv   u = k,  x = q,  y = do   late (from the last token back), Z = dS
//   dk   u = v,  x = do, y = q    late, Z = dS^T
// so that one kernel serves all.  In chunks of C tokens (places i, j in the chunk, n of them there):
//   early  row_i = g^{i+1} Z^T u_i + sum_{j <= i} g^{i-j} (u_i . x_j) y_j      Z' = g^n Z + sum_j g^{n-1-j} x_j y_j^T
//   late   row_i = g^{n-1-i} Z^T u_i + sum_{j >= i} g^{j-i} (u_i . x_j) y_j    Z' = g^n Z + sum_j g^{j+1} x_j y_j^T
// (in a late walk Z is what reaches the chunk's last token, E, which it uses before it is decayed).  The
// chunks of a sequence start at its first token in both.
#pragma once

#include "common.cuh"

namespace dgc {

struct Heads { const void* p; int64_t ld, head; };

struct Walk {
  Heads u, x, y;
  void* out;
  int64_t out_ld, out_head;
  const float* z_in;     // states before the walk; NULL: 0
  float* z_out;          // states after it; may be NULL
  int32_t du, dy;        // lengths of u (and x) and of y (and the rows)
  int32_t late, turned;  // turned: z_in is kept as [dy][du], else [du][dy]
  float w_row, w_near, w_x;   // factors of Z^T u, of the sum over the chunk, of x on its way to Z
  int32_t dout;               // 1: u is the gradient of the output, 2: x is
};

constexpr int kMaxWalks = 3;
struct WalkArgs {
  Walk w[kMaxWalks];
  const float* decay;
  const int32_t* seq_start;
  int32_t tokens, seqs, seq_len, heads;
  int32_t part;          // tokens of a part (a multiple of 128), or 0: whole sequences
  int32_t slices;        // blocks that share the rows' dy
  const uint8_t* dout_tops;   // [heads][tokens], in DGC_F16: the biased exponent of the largest finite |dout|, 1 at the least; NULL: not known
  int32_t longest_first; // whole sequences, taken in the order of their lengths
};

// Which sequence and which of its tokens an item is.  Sequences are cut into parts; part 0 of sequence s is
// item floor(start / part) + s, which leaves room for all parts of those before it:
// ceil(length / part) <= floor(end / part) - floor(start / part) + 1.
struct Item { int s, first, len, seq_first, seq_len; };
__device__ __forceinline__ void sequence_of(const WalkArgs& a, int s, int& first, int& len) {
  if (a.seq_start) {   // offsets are clamped: a damaged table cannot lead outside the tensors
    const int lo = min(max(__ldg(a.seq_start + s), 0), a.tokens);
    const int hi = min(max(__ldg(a.seq_start + s + 1), lo), a.tokens);
    first = lo;
    len = hi - lo;
  } else {
    first = s * a.seq_len;
    len = a.seq_len;
  }
}
// The sequence that is `place`-th in length (the longest first, the first first among equals): blocks start
// in this order, so that the last to start have little left to do.  For a whole block.
constexpr int kSorted = 256;
__device__ __forceinline__ int by_length(const WalkArgs& a, int place) {
  __shared__ int lens[kSorted];
  __shared__ int found;
  for (int t = threadIdx.x; t < a.seqs; t += blockDim.x) {
    int first;
    sequence_of(a, t, first, lens[t]);
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
__device__ __forceinline__ int first_item(const WalkArgs& a, int s) {
  int first, len;
  sequence_of(a, s, first, len);
  return first / a.part + s;
}
__device__ __forceinline__ Item item_of(const WalkArgs& a, int item) {
  Item it{};
  if (!a.part) {
    it.s = a.longest_first ? by_length(a, item) : item;
    sequence_of(a, it.s, it.seq_first, it.seq_len);
    it.first = it.seq_first;
    it.len = it.seq_len;
    return it;
  }
  int lo = 0, hi = a.seqs - 1;   // the last sequence whose first item is not behind this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first_item(a, mid) <= item) lo = mid;
    else hi = mid - 1;
  }
  it.s = lo;
  sequence_of(a, lo, it.seq_first, it.seq_len);
  const int64_t off = (int64_t)(item - (it.seq_first / a.part + lo)) * a.part;
  it.first = it.seq_first;
  if (off >= 0 && off < it.seq_len) {
    it.first += (int)off;
    it.len = min(a.part, it.seq_len - (int)off);
  }
  return it;
}

int32_t attention_waits_out(int* count);   // of the attention's kernels, see tensor.cuh

// log2 of a decay, finite: decays below 2^-1000 (0) forget everything at once, and 0^0 is 1.
__device__ __forceinline__ float log_decay(const float* decay, int h) { return fmaxf(log2f(__ldg(decay + h)), -1000.0f); }

}  // namespace dgc
