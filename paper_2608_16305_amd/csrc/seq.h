// Sequences laid one after the other in the rows of a matrix (mtgnn_seqs), as the convolution and the scan walk them.
#pragma once

#include "common.h"

namespace mtgnn {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// e^x on the hardware's base-2 exponential, with the part of x log2 e that its float32 product loses: exact to a unit
// of the last place or two (the product alone is off by |x| units).  x <= 0.
__device__ __forceinline__ float exp_neg(float x) {
  const float y = x < -150.f ? -150.f : x;   // e^-150 is 0; a NaN stays one
  const float t = y * LOG2E, r = fmaf(y, 1.9259629911266175e-8f, fmaf(y, LOG2E, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, r * LN2, e);
}
// softplus(u) = max(u, 0) + log1p(e^-|u|).  log1p(v) = 2 atanh(s) with s = v / (2 + v) <= 1/3; atanh(s) / s as the
// polynomial in s^2 that a Chebyshev fit over [0, 1/9] gives (8e-9 off at most): exact to a few units of the last
// place for every v, small ones too, where log(1 + v) has lost v's low bits.
__device__ __forceinline__ float softplus_(float u) {
  const float v = exp_neg(-fabsf(u));
  const float s = v * __builtin_amdgcn_rcpf(2.f + v), q = s * s;
  float p = 0.1408732831478119f;
  p = fmaf(p, q, 0.1398070901632309f);
  p = fmaf(p, q, 0.20012426376342773f);
  p = fmaf(p, q, 0.3333315849304199f);
  p = fmaf(p, q, 1.f);
  return fmaf(2.f * s, p, fmaxf(u, 0.f));   // a NaN stays one through v
}
__device__ __forceinline__ float silu_(float p) { return p * sigmoid_hw(p); }
__device__ __forceinline__ float dsilu_(float p) {
  const float s = sigmoid_hw(p);
  return s * fmaf(p, 1.f - s, 1.f);
}
// act and its derivative for mtgnn_act `act` (uniform).
__device__ __forceinline__ float act_(int act, float p) {
  if (act == MTGNN_ACT_SILU) return silu_(p);
  if (act == MTGNN_ACT_RELU) return p < 0.f ? 0.f : p;   // a NaN stays one
  if (act == MTGNN_ACT_GELU) return 0.5f * p * (1.f + erff(p * 0.70710678118654752f));
  return p;
}
__device__ __forceinline__ float dact_(int act, float p) {
  if (act == MTGNN_ACT_SILU) return dsilu_(p);
  if (act == MTGNN_ACT_RELU) return p > 0.f ? 1.f : 0.f;
  if (act == MTGNN_ACT_GELU)
    return 0.5f * (1.f + erff(p * 0.70710678118654752f)) + p * expf(-0.5f * p * p) * 0.3989422804014327f;
  return 1.f;
}

struct Seqs {
  const int32_t *off, *n_seq, *slot;
  int64_t max_seq, max_rows, n_slots;
};
inline Seqs seqs_of(const mtgnn_seqs* q) {
  return Seqs{q->off, q->n_seq, q->slot, q->max_seq, q->max_rows, q->n_slots};
}

// The rows of all sequences: [lo, hi), and the number of sequences.
struct SeqRange {
  int n, lo, hi;
};
__device__ __forceinline__ SeqRange seq_range(const Seqs& q) {
  SeqRange r{(int)q.max_seq, 0, 0};
  if (q.n_seq) {
    const int c = *q.n_seq;
    r.n = c < 0 ? 0 : c < r.n ? c : r.n;
  }
  if (r.n > 0) {
    const int lo = q.off[0], hi = q.off[r.n];
    r.lo = lo < 0 ? 0 : lo;
    r.hi = hi < (int)q.max_rows ? hi : (int)q.max_rows;
  }
  return r;
}

// The sequence that holds row t (lo <= t < hi) and its rows [beg, end).  Found by the whole wave: each round
// compares 64 evenly spaced starts at once, so 262,144 sequences take three dependent reads, not eighteen.
struct SeqAt {
  int s, beg, end;
};
__device__ __forceinline__ SeqAt seq_find(const int32_t* off, int n, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, cnt = n;
  while (cnt > 1) {
    const int step = (cnt + 63) >> 6, i = lane * step;
    const bool le = i < cnt && off[lo + (i < cnt ? i : 0)] <= t;
    const int k = __popcll(__ballot(le));
    const int j = (k > 0 ? k - 1 : 0) * step;
    lo += j;
    cnt = cnt - j < step ? cnt - j : step;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return SeqAt{lo, off[lo], off[lo + 1]};
}
// A walk over the sequences that have rows.  The wave holds 64 consecutive starts (lane l: off[w0 + l], w0 <= s) and their
// slots and reads them from its lanes: a start costs a register read, not a dependent trip to memory.  Sequences without
// rows are passed over at once, however many they are: in the window by comparing all its starts, else by a search.  (One
// after the other they took 0.12 us each.)
struct SeqWalk {
  const int32_t *off, *slot;
  int64_t n_slots;
  int n, s, beg, end, w0, v_off, v_slot;
  __device__ __forceinline__ SeqWalk(const Seqs& q, const SeqRange& r, int t) : off(q.off), slot(q.slot), n_slots(q.n_slots), n(r.n) {
    const SeqAt a = seq_find(off, n, t);
    s = a.s;
    beg = a.beg;
    end = a.end;
    window(s);
  }
  __device__ __forceinline__ void window(int at) {
    const int lane = threadIdx.x & 63;
    w0 = at < 0 ? 0 : at;
    v_off = off[min(w0 + lane, n)];
    v_slot = slot ? slot[min(w0 + lane, n - 1)] : w0 + lane;
  }
  // To the next (previous) sequence that has rows: the one that holds the row behind this one's last (before its first).
  // Where there is none, to the last (first) of all, as one without rows.  Whatever the offsets hold, a step gets further
  // or to that end, and s stays below n.
  __device__ __forceinline__ void next() {
    beg = end;
    uint64_t behind = __ballot(v_off > beg);
    if (!behind) {
      window(seq_find(off, n, beg).s);
      behind = __ballot(v_off > beg);
    }
    s = n - 1;
    if (!behind) return;
    const int j = __builtin_ctzll(behind);
    s = w0 + (j > 0 ? j - 1 : 0);
    end = __builtin_amdgcn_readlane(v_off, j);
  }
  __device__ __forceinline__ void prev() {
    end = beg;
    uint64_t before = s - w0 < 64 ? __ballot(v_off < end) : 0;
    if (!before) {
      window(seq_find(off, n, end - 1).s - 63);
      before = __ballot(v_off < end);
    }
    const int j = before ? 63 - __builtin_clzll(before) : 0;
    s = before ? min(w0 + j, n - 1) : 0;
    beg = before ? __builtin_amdgcn_readlane(v_off, j) : 0;
    end = before ? end : 0;
  }
  // The table row of the sequence, or -1: no carried state.
  __device__ __forceinline__ int64_t row() {
    if (s < w0 || s > w0 + 63) window(s - 32);
    const int k = __builtin_amdgcn_readlane(v_slot, s - w0);
    return k >= 0 && k < n_slots ? k : -1;
  }
};
// The table row of sequence (or single row) s, or -1: no carried state.
__device__ __forceinline__ int64_t seq_slot(const int32_t* slot, int64_t n_slots, int64_t s) {
  const int64_t k = slot ? (int64_t)slot[s] : s;
  return k >= 0 && k < n_slots ? k : -1;
}

namespace {

// Column sums of the chunks' shares part[chunk][cols] in order, into up to three tensors of n0, n1, cols - n0 - n1
// columns (each may be NULL); a chunk is `ch` rows, and only those with rows have a share (q.off NULL: `n_parts` shares
// all have one).  16 columns a block, 16 threads to each.
__global__ __launch_bounds__(256) void k_sum_parts(Seqs q, int ch, int n_parts, const float* part, int64_t cols,
                                                   int64_t n0, float* out0, int64_t n1, float* out1, float* out2) {
  __shared__ float s[16][17];
  int c0 = 0, c1 = n_parts;
  if (q.off) {
    const SeqRange r = seq_range(q);
    c0 = r.lo < r.hi ? r.lo / ch : 0;
    c1 = r.lo < r.hi ? (r.hi - 1) / ch + 1 : 0;
  }
  const int j = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int64_t col = (int64_t)blockIdx.x * 16 + j;
  float v = 0.f;
  if (col < cols)
    for (int c = c0 + k; c < c1; c += 16) v += part[c * cols + col];
  s[k][j] = v;
  __syncthreads();
  if (k == 0 && col < cols) {
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += s[i][j];
    if (col < n0) {
      if (out0) out0[col] = v;
    } else if (col < n0 + n1) {
      if (out1) out1[col - n0] = v;
    } else if (out2) {
      out2[col - n0 - n1] = v;
    }
  }
}

}  // namespace

}  // namespace mtgnn
