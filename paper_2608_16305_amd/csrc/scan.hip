// Selective state space scan over ragged sequences: whole sequences, their backward, and single rows.
//
//   dt = softplus(delta + delta_bias),  h_t = exp(dt A) h_(t-1) + dt B x,  y = (C . h + D x) silu(z)
//
// per channel and state.  The recurrence is linear in h, so rows are cut into chunks that are worked on at once:
//   k_scan_local   each chunk's last state from zeros (or from the last start of a sequence in it) and the decay
//                  over the chunk, exp(A sum dt): one exponential per chunk, not a product of many;
//   k_scan_carry   the state that enters each chunk, over the chunks in order;
//   k_scan_out     each chunk again from the state that enters it, now with y.
// A chunk is a range of rows, whatever sequences they belong to: a start of a sequence inside it replaces the
// state, so one sequence of 100,000 rows and 100,000 sequences of one row are the same amount of work per wave.
// One chunk (few rows) needs k_scan_out alone.
//
// Forward kernels: a wave has 64 channels of one group, a lane one channel and all its states, so the sum over the states
// and everything of a row and channel stay in its lane.  B and C are the same for all lanes: read by scalar loads
// into scalar registers, which the products take as they are, where a row is whole words of a supported
// number of states, else staged in LDS and read by all lanes at once.
// Backward: the sums that dB and dC need are over channels.  There a lane has four channels and 4 (2, 1) states, lane l the
// channels 4 (l / 4) .. + 3, wave w the states 16 w .. 16 w + 15: sums over states are over four lanes, those over
// channels over registers first and then 16 lanes, where a channel a lane would take all 64.
//
// Vector instructions bound it: per row, channel and state an exponential (four times an ordinary instruction's
// cycles) and three or four products and sums, once in k_scan_local and once in k_scan_out, against 8 bytes per row and
// channel in bfloat16.  Measured with 16 states, bfloat16, gate and skip: 32,768 rows x 2,048 of 5 sequences take
// 224 (local) + 14 (carry) + 363 us (out), 1.07e9 exponentials in each of local and out, 70 to 85% of the cycles issue vector
// instructions; in out some of them move scalar registers that B and C leave no room for.  Training, 16,384 x 1,024:
// 65 + 15 + 112 forward, backward 82 + 15 + 347 + 22 for the sums.  8,000 rows x 100 of 6,000 sequences: 14 + 17 + 26 us, a
// chain of dependent reads (count, search, offsets, rows, states), and the carry's latency.
#include <algorithm>

#include "bf16_split.h"
#include "ops.h"
#include "seq.h"

namespace mtgnn {

namespace {

constexpr int TT = 8;      // rows of a tile, and of a checkpoint of the forward
constexpr int CT = 64;     // channels of a block

struct ScanP {
  Seqs q;
  const void *x, *delta, *B, *C, *z;
  int64_t ldx, ldd, ldB, ldC, ldz;
  const float *A, *D, *bias;
  int d, n, groups, per, tpg, nct, softplus;   // per: channels of a group; tpg: tiles of a group; nct: tiles in all
  int ch, nchunk, vec;                         // rows of a chunk; vec: four channels of a state row are 16-byte aligned
  const float* st_in;
  float* st_out;
  void* y;
  int64_t ldy;
  float *hs, *init;                            // saved: checkpoints [rows / 8][n][d], first states [max_seq][n][d]
  int32_t* carried;                            // saved: whether there are first states
  float *E, *sumdt;                            // [nchunk][n][d], [nchunk][d]
  int32_t* flag;                               // [nchunk]
  // [nchunk][n][d] or NULL: where one table is read and written, the first state of a sequence that goes on in the
  // next chunk.  Another block writes its slot, maybe before this one has read it; a sequence that ends in
  // its chunk is read and written by the same threads.
  float* first;
};
struct ScanG {
  const float* dy;
  int64_t lddy;
  float *dx, *ddelta, *dB, *dC, *dz;
  int64_t lddx, lddd, lddB, lddC, lddz;
  float *part, *bc;                            // [nchunk][n + 2][d]; [nct][rows][2][n] (one tile per group: unused)
};

// What a chunk hands on: its own state plus the decayed one that enters; its own alone (a sequence starts in
// it); nothing (the next chunk starts with a sequence, or there are no rows).
enum { CARRY_ADD = 0, CARRY_OWN = 1, CARRY_NONE = 2 };

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int QUAD_XOR1 = 0xB1, QUAD_XOR2 = 0x4E, ROW_ROR4 = 0x124, ROW_ROR8 = 0x128;

// Lane j of each four lanes gets the sum of v[j] over the four.
__device__ __forceinline__ float quad_sums(const float (&v)[4]) {
  const bool b0 = threadIdx.x & 1, b1 = threadIdx.x & 2;
  const float r0 = (b0 ? v[1] : v[0]) + dpp<QUAD_XOR1>(b0 ? v[0] : v[1]);
  const float r1 = (b0 ? v[3] : v[2]) + dpp<QUAD_XOR1>(b0 ? v[2] : v[3]);
  return (b1 ? r1 : r0) + dpp<QUAD_XOR2>(b1 ? r0 : r1);
}

// Four channels' values of one state row.  vec: p is 16-byte aligned wherever all four exist.
__device__ __forceinline__ void load4(const float* p, int left, bool vec, float (&v)[4]) {
  if (vec && left >= 4) {
    const float4 f = *(const float4*)p;
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    return;
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = c < left ? p[c] : 0.f;
}
__device__ __forceinline__ void store4(float* p, int left, bool vec, float a, float b, float c, float d) {
  if (vec && left >= 4) {
    *(float4*)p = make_float4(a, b, c, d);
    return;
  }
  if (left > 0) p[0] = a;
  if (left > 1) p[1] = b;
  if (left > 2) p[2] = c;
  if (left > 3) p[3] = d;
}

// The value, but not one that is known outside: the addresses that are made from it are made where they are used,
// where otherwise a loop's 2 N of them would be kept in scalar registers that B and C need.
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+s"(v));
  return v;
}

// Where a thread stands.
template <int SPL, int NB>
struct Place {
  static constexpr int NP = 4 * SPL * NB;
  int lane, wid, cb, n0, g, ch0, left;   // cb: first of its channels in the block; left: channels of the group from ch0
  __device__ __forceinline__ Place(const ScanP& p, int tile) {
    lane = threadIdx.x & 63;
    wid = NB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    cb = lane & ~3;
    n0 = wid * 4 * SPL + (lane & 3) * SPL;
    g = tile / p.tpg;
    const int in = (tile % p.tpg) * CT;
    ch0 = g * p.per + in;
    left = min(CT, p.per - in);
  }
  // h of state table row `row` (of n x d floats, fewer than 2^26)
  __device__ __forceinline__ void load(const ScanP& p, const float* tab, int64_t row, float (&h)[4][SPL]) const {
    const int d = opaque(p.d);
    const float* q = tab + row * p.n * d + ch0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (n0 + s < p.n) load4(q + (uint32_t)((n0 + s) * d + cb), left - cb, p.vec, v);
#pragma unroll
      for (int c = 0; c < 4; ++c) h[c][s] = v[c];
    }
  }
  __device__ __forceinline__ void store(const ScanP& p, float* tab, int64_t row, const float (&h)[4][SPL]) const {
    const int d = opaque(p.d);
    float* q = tab + row * p.n * d + ch0;
#pragma unroll
    for (int s = 0; s < SPL; ++s)
      if (n0 + s < p.n)
        store4(q + (uint32_t)((n0 + s) * d + cb), left - cb, p.vec, h[0][s], h[1][s], h[2][s], h[3][s]);
  }
  __device__ __forceinline__ void decay(const ScanP& p, float (&A2)[4][SPL]) const {   // A log2 e
    load(p, p.A, 0, A2);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int s = 0; s < SPL; ++s) A2[c][s] *= LOG2E;
  }
};

__device__ __forceinline__ void zero_state(float* h, int n) {
  for (int i = 0; i < n; ++i) h[i] = 0.f;
}

// A tile's B or C rows (float, zero past the n states) into dst[TT][NP]; rows clamped to the last.
template <typename T, int NP, int NT>
__device__ __forceinline__ void stage_states(const void* src, int64_t ld, int n, int col0, int row, int last,
                                             float* dst) {
  for (int e = threadIdx.x; e < TT * NP; e += NT) {
    const int i = e / NP, s = e % NP;
    const float v = Elem<T>::load((const T*)src, (int64_t)min(row + i, last) * ld + col0 + min(s, n - 1));
    dst[e] = s < n ? v : 0.f;
  }
}

__device__ __forceinline__ float step_size(const ScanP& p, float u) { return p.softplus ? softplus_(u) : u; }
// A tile's step sizes, and its gates, in place.  One branch for all of them, so that the rows after it are one run of
// instructions in which B and C are requested ahead.
__device__ __forceinline__ void step_sizes(const ScanP& p, float bias, float (&u)[TT]) {
#pragma unroll
  for (int i = 0; i < TT; ++i) u[i] += bias;
  if (p.softplus) {
#pragma unroll
    for (int i = 0; i < TT; ++i) u[i] = softplus_(u[i]);
  }
}
__device__ __forceinline__ void gates(const ScanP& p, float (&z)[TT]) {
  if (p.z) {
#pragma unroll
    for (int i = 0; i < TT; ++i) z[i] = silu_(z[i]);
  }
}

template <int SPL>
__device__ __forceinline__ void lds_get(const float* p, float (&v)[SPL]) {
  if constexpr (SPL == 4) {
    const float4 f = *(const float4*)p;
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else if constexpr (SPL == 2) {
    const float2 f = *(const float2*)p;
    v[0] = f.x; v[1] = f.y;
  } else {
    v[0] = p[0];
  }
}

template <int SPL>
__device__ __forceinline__ void lds_put(float* p, const float (&v)[SPL]) {
  if constexpr (SPL == 4) *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  else if constexpr (SPL == 2) *(float2*)p = make_float2(v[0], v[1]);
  else p[0] = v[0];
}

// Which rows of chunk c exist.
__device__ __forceinline__ void chunk_rows(const ScanP& p, const SeqRange& r, int c, int& t0, int& t1) {
  const int64_t a = (int64_t)c * p.ch;
  t0 = (int)(a > r.lo ? a : r.lo);
  t1 = (int)(a + p.ch < r.hi ? a + p.ch : r.hi);
}

// ------------------------------------------------------------------ forward

// A lane's channel and its N states (of more than 32, each of two waves has half).
struct Lane {
  int g, col0, n0, wave;
  uint32_t col;     // of the lane, in its tile's first .. last channel
  bool mine;
  __device__ __forceinline__ Lane(const ScanP& p, int tile, int N) {
    const int lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    n0 = wave * N;
    g = tile / p.tpg;
    const int in = (tile % p.tpg) * CT;
    col0 = g * p.per + in;
    mine = in + lane < p.per;
    col = mine ? lane : 0;
  }
  template <typename T>
  __device__ __forceinline__ float at(const void* m, int64_t ld, int64_t row) const {   // m[row][channel]
    return Elem<T>::load((const T*)m + row * ld + col0, col);
  }
  template <int N>
  __device__ __forceinline__ void load(const ScanP& p, const float* tab, int64_t row, float (&h)[N]) const {
    const int64_t step = opaque(p.d);
    const float* q = tab + (row * p.n + n0) * step + col0;
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = n0 + i < p.n ? q[i * step + col] : 0.f;
  }
  template <int N>
  __device__ __forceinline__ void store(const ScanP& p, float* tab, int64_t row, const float (&h)[N]) const {
    const int64_t step = opaque(p.d);
    float* q = tab + (row * p.n + n0) * step + col0;
    if (!mine) return;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (n0 + i < p.n) q[i * step + col] = h[i];
  }
  template <int N>
  __device__ __forceinline__ void decay(const ScanP& p, float (&A2)[N]) const {   // A log2 e
    load(p, p.A, 0, A2);
#pragma unroll
    for (int i = 0; i < N; ++i) A2[i] *= LOG2E;
  }
};

// B or C of a row, the same in every lane.  SC: by scalar loads (N words of float, or N / 2 of bfloat16 pairs; the matrix
// is not written while the kernel runs); else from the tile staged in LDS.
template <typename T, int N, bool SC>
struct States {
  static constexpr int WORDS = SC ? 4 : TT * N;
  const T* m;
  int64_t ld;
  int n;
  float* lds;
  __device__ __forceinline__ States(const void* src, int64_t ld_, int n_, const Lane& me, float* lds_)
      : m((const T*)src + me.g * n_ + me.n0), ld(ld_), n(n_ - me.n0), lds(lds_ + me.wave * WORDS) {}
  __device__ __forceinline__ void stage(int row, int last) const {
    if constexpr (!SC) {
      for (int e = threadIdx.x & 63; e < TT * N; e += 64) {
        const int i = e / N, s = e % N;
        const float v = Elem<T>::load(m, (int64_t)min(row + i, last) * ld + min(s, n - 1));
        lds[e] = s < n ? v : 0.f;
      }
    }
  }
  // Sixteen states at a time (more of B and C have no registers): their words as read, and their values.
  static constexpr int M = N < 16 ? N : 16, PARTS = N / M;
  struct Raw {
    uint32_t w[SC ? M * sizeof(T) / 4 : 1];
  };
  __device__ __forceinline__ Raw fetch(int row, int part) const {
    Raw r;
    if constexpr (SC) {
      const auto q = (const __attribute__((address_space(4))) uint32_t*)(uintptr_t)(m + row * ld + part * M);
#pragma unroll
      for (int k = 0; k < (int)(M * sizeof(T) / 4); ++k) r.w[k] = q[k];
    }
    return r;
  }
  __device__ __forceinline__ void values(const Raw& r, int i, int part, float (&v)[M]) const {   // row i of the tile
    if constexpr (SC) {
#pragma unroll
      for (int k = 0; k < M; ++k) {
        if constexpr (sizeof(T) == 4) v[k] = __uint_as_float(r.w[k]);
        else v[k] = __uint_as_float(k % 2 ? r.w[k / 2] & 0xffff0000u : r.w[k / 2] << 16);
      }
    } else {
#pragma unroll
      for (int k = 0; k < M; k += 4) {
        const float4 f = *(const float4*)(lds + i * N + part * M + k);
        v[k] = f.x; v[k + 1] = f.y; v[k + 2] = f.z; v[k + 3] = f.w;
      }
    }
  }
};
// f(row of the tile, part of the states, words of B (and C) for it), over all rows of a tile from FIRST in steps of
// STEP (1 or -1), the next part's words requested before this one's work: the compiler would wait for each where it
// is used, or bring all of a tile forward and run out of registers.
template <int STEP, class S, class F>
__device__ __forceinline__ void over_tile(const S& a, const S& b, bool two, int tb, F f) {
  constexpr int FIRST = STEP > 0 ? 0 : TT - 1;
  typename S::Raw ra = a.fetch(tb + FIRST, 0), rb = two ? b.fetch(tb + FIRST, 0) : ra;
#pragma unroll
  for (int q = 0; q < TT * S::PARTS; ++q) {
    const int i = FIRST + STEP * (q / S::PARTS), part = q % S::PARTS;
    const int qn = q + 1 < TT * S::PARTS ? q + 1 : q;
    const int in = FIRST + STEP * (qn / S::PARTS), pn = qn % S::PARTS;
    const typename S::Raw na = a.fetch(tb + in, pn), nb = two ? b.fetch(tb + in, pn) : na;
    f(i, part, ra, rb);
    __builtin_amdgcn_sched_barrier(0);
    ra = na;
    rb = nb;
  }
}
template <typename T>
__device__ __forceinline__ void put(T* row, uint32_t col, float v) {
  if constexpr (sizeof(T) == 2) row[col] = (uint16_t)cvt2_bf16(v, v);
  else row[col] = v;
}
template <int N>
__device__ __forceinline__ void zero(float (&h)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) h[i] = 0.f;
}

template <typename T, int N, int NW, bool SC>
__global__ __launch_bounds__(64 * NW) void k_scan_local(ScanP p) {
  __shared__ __align__(16) float s_B[NW * States<T, N, SC>::WORDS];
  const int c = blockIdx.x / p.nct, tile = blockIdx.x % p.nct;
  const Lane me(p, tile, N);
  const States<T, N, SC> B(p.B, p.ldB, p.n, me, s_B);
  const SeqRange r = seq_range(p.q);
  int t0, t1;
  chunk_rows(p, r, c, t0, t1);
  int flag = CARRY_NONE;
  SeqAt at{0, 0, 0};
  if (t0 < t1) {
    at = seq_find(p.q.off, r.n, t1 - 1);
    if (at.end > t1) flag = at.beg >= t0 ? CARRY_OWN : CARRY_ADD;
  }
  if (tile == 0 && threadIdx.x == 0) p.flag[c] = flag;
  if (flag == CARRY_NONE) return;
  float A2[N], h[N];
  me.decay(p, A2);
  zero(h);
  int t = t0;
  if (flag == CARRY_OWN) {
    t = at.beg;
    const int64_t k = p.st_in ? seq_slot(p.q.slot, p.q.n_slots, at.s) : -1;
    if (k >= 0) me.load(p, p.st_in, k, h);
    if (p.first) me.store(p, p.first, c, h);
  }
  const float bias = p.bias ? p.bias[me.col0 + me.col] : 0.f;
  float sum = 0.f;
  for (; t < t1; t += TT) {
    float u[TT], x[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      const int row = min(t + i, t1 - 1);
      u[i] = me.at<T>(p.delta, p.ldd, row);
      x[i] = me.at<T>(p.x, p.ldx, row);
    }
    B.stage(t, t1 - 1);
    if constexpr (!SC) __syncthreads();
    step_sizes(p, bias, u);
    using S = States<T, N, SC>;
    const auto part = [&](int i, int k, const typename S::Raw& rb, const typename S::Raw&) {
      const float dt = u[i], dx = dt * x[i];
      if (k == 0) sum += dt;
      float b[S::M];
      B.values(rb, i, k, b);
#pragma unroll
      for (int s = 0; s < S::M; ++s) {
        float& hs = h[k * S::M + s];
        hs = fmaf(__builtin_amdgcn_exp2f(dt * A2[k * S::M + s]), hs, dx * b[s]);
      }
    };
    if (t + TT <= t1) {
      over_tile<1>(B, B, false, t, part);
    } else {
#pragma unroll
      for (int i = 0; i < TT; ++i) {
        if (t + i >= t1) break;
#pragma unroll
        for (int k = 0; k < S::PARTS; ++k) {
          const typename S::Raw rb = B.fetch(t + i, k);
          part(i, k, rb, rb);
        }
      }
    }
    if constexpr (!SC) __syncthreads();
  }
  me.store(p, p.E, c, h);
  if (me.mine && me.wave == 0) p.sumdt[(int64_t)c * p.d + me.col0 + me.col] = sum;
}

// own + 2^s h.  The power's whole part goes to h's exponent: past float32's range it still meets a small h as it would row
// after row, and a zero one stays zero (an infinite decay times zero is NaN).  h spans 2^277, so s past +-1000 is as at
// it; an infinite one is an infinite step's, 2^s then 0 or infinite (NaN with an infinite or a zero h, as there); where s
// is NaN own is too.  1 us of k_scan_carry's 14 against a product with exp2(s).
__device__ __forceinline__ float carried(float s, float h, float own) {
  const float t = __builtin_amdgcn_fmed3f(s, -1000.f, 1000.f);
  const float e = __builtin_amdgcn_exp2f(fabsf(s) == INFINITY ? s : __builtin_amdgcn_fractf(t));
  return fmaf(e, ldexpf(h, (int)floorf(t)), own);
}

// The state that enters each chunk, in place of E.  back: the same for the flow that runs from the last chunk to the
// first.  A block has 1024 / RUNS states and channels; each of RUNS threads to one takes a run of chunks, once for
// what the run hands on, h -> own + decay h, and, after a scan over the runs, once with what enters it.  (One
// thread over all chunks waited for memory 127 times in turn at 1,013 chunks: 144 us, against 16.)  Latency bounds it.
// 64 runs from 256 chunks on, else 16: 16.3 against 36 us at 1,013 chunks x 1,600; 29.7 against 13.4 at 128 x 32,768 (1 us
// less each than now, with decays in place of their exponents).
template <int RUNS>
__global__ __launch_bounds__(1024) void k_scan_carry(ScanP p, int back) {
  constexpr int RUN_COLS = 1024 / RUNS;
  // s_t: the sum of dt over a run, whose decay what enters the run passes with.  NaN: nothing passes (a NaN of the inputs'
  // own: nothing that matters, since the run's state is NaN then).
  __shared__ float s_h[RUNS][RUN_COLS + 1], s_t[RUNS][RUN_COLS + 1];
  const int64_t nd = (int64_t)p.n * p.d;
  const int j = threadIdx.x % RUN_COLS, run = threadIdx.x / RUN_COLS;
  const int64_t i = min((int64_t)blockIdx.x * RUN_COLS + j, nd - 1);
  const bool mine = (int64_t)blockIdx.x * RUN_COLS + j < nd;
  const int ch = (int)(i % p.d);
  const float A2 = p.A[i] * LOG2E;
  const int len = (p.nchunk + RUNS - 1) / RUNS, k0 = run * len, k1 = min(p.nchunk, k0 + len);
  const auto walk = [&](float& h, float& t, bool write) {
    constexpr int U = 8;
    for (int k = k0; k < k1; k += U) {
      float e[U], sd[U];
      int f[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = min(k + u, k1 - 1), c = back ? p.nchunk - 1 - v : v;
        e[u] = p.E[c * nd + i];
        sd[u] = p.sumdt[(int64_t)c * p.d + ch];
        f[u] = p.flag[c];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k + u >= k1) break;
        const int c = back ? p.nchunk - 1 - (k + u) : k + u;
        if (write && mine) p.E[c * nd + i] = h;
        const float next = carried(A2 * sd[u], h, e[u]);
        h = f[u] == CARRY_ADD ? next : f[u] == CARRY_OWN ? e[u] : 0.f;
        t = f[u] == CARRY_ADD ? t + sd[u] : NAN;
      }
    }
  };
  float h = 0.f, t = 0.f;
  walk(h, t, false);
  s_h[run][j] = h;
  s_t[run][j] = t;
  __syncthreads();
  for (int o = 1; o < RUNS; o <<= 1) {
    const float ph = run >= o ? s_h[run - o][j] : 0.f, pt = run >= o ? s_t[run - o][j] : 0.f;
    __syncthreads();
    h = t == t ? carried(A2 * t, ph, h) : h;
    t += pt;
    s_h[run][j] = h;
    s_t[run][j] = t;
    __syncthreads();
  }
  h = run > 0 ? s_h[run - 1][j] : 0.f;
  walk(h, t, true);
}

// PAD: there are fewer than N NW states (never by scalar loads).  Those past the last hold zero times what comes in, NaN
// where that is infinite, and then for good: tiles in which something is go the way of the mixed ones, where such a row's
// are put back to zero.  1 to 2% of a call; 3 to 6% if every row of every tile looks.
template <typename T, int N, int NW, bool SC, bool PAD>
__global__ __launch_bounds__(64 * NW) void k_scan_out(ScanP p) {
  __shared__ __align__(16) float s_B[NW * States<T, N, SC>::WORDS], s_C[NW * States<T, N, SC>::WORDS];
  const int c = blockIdx.x / p.nct, tile = blockIdx.x % p.nct;
  const Lane me(p, tile, N);
  const States<T, N, SC> B(p.B, p.ldB, p.n, me, s_B), C(p.C, p.ldC, p.n, me, s_C);
  __shared__ float s_y[NW > 1 ? NW : 1][NW > 1 ? TT : 1][64];
  if (p.carried && blockIdx.x == 0 && threadIdx.x == 0) *p.carried = p.st_in != nullptr;
  const SeqRange r = seq_range(p.q);
  int t0, t1;
  chunk_rows(p, r, c, t0, t1);
  if (t0 >= t1) return;
  SeqWalk at(p.q, r, t0);
  float A2[N], h[N];
  me.decay(p, A2);
  zero(h);
  if (at.beg < t0) me.load(p, p.E, c, h);
  const float bias = p.bias ? p.bias[me.col0 + me.col] : 0.f, D = p.D ? p.D[me.col0 + me.col] : 0.f;
  for (int tb = t0 / TT * TT; tb < t1; tb += TT) {
    float u[TT], x[TT], z[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      const int row = min(max(tb + i, t0), t1 - 1);
      u[i] = me.at<T>(p.delta, p.ldd, row);
      x[i] = me.at<T>(p.x, p.ldx, row);
      z[i] = p.z ? me.at<T>(p.z, p.ldz, row) : 1.f;
    }
    if constexpr (NW > 1) __syncthreads();   // the last tile's s_y is read, and every wave has its rows: y may be one of them
    B.stage(tb, t1 - 1);
    C.stage(tb, t1 - 1);
    if constexpr (!SC) __syncthreads();
    step_sizes(p, bias, u);
    bool tame = true;
    if constexpr (PAD) {
      float all = 0.f;   // not finite where a term is not
#pragma unroll
      for (int i = 0; i < TT; ++i) all = fmaf(u[i], x[i], all);
      tame = !__any(!(fabsf(all) < INFINITY));
    }
    gates(p, z);
    using S = States<T, N, SC>;
    float y[2];
    const auto part_of = [&](auto keep, int i, int k, const typename S::Raw& rb, const typename S::Raw& rc) {   // z[i] becomes y
      const float dt = u[i], dx = dt * x[i];
      const float skip = p.D && (NW == 1 || me.wave == 0) ? D * x[i] : 0.f;   // (no D: not 0 times an x that may be infinite)
      if (k == 0) {
        y[0] = skip;
        y[1] = 0.f;
      }
      float b[S::M], cc[S::M];
      B.values(rb, i, k, b);
      C.values(rc, i, k, cc);
#pragma unroll
      for (int s = 0; s < S::M; ++s) {
        float& hs = h[k * S::M + s];
        hs = fmaf(__builtin_amdgcn_exp2f(dt * A2[k * S::M + s]), hs, dx * b[s]);
        y[s & 1] = fmaf(hs, cc[s], y[s & 1]);
      }
      if (k == S::PARTS - 1) {
        if constexpr (decltype(keep)::value) {
          if (!tame && __any(!(y[0] + y[1] == y[0] + y[1]))) {   // NaN: the sum again, without them
            y[0] = skip;
            y[1] = 0.f;
#pragma unroll
            for (int q = 0; q < N; ++q) {
              if (q >= C.n) h[q] = 0.f;
              y[q & 1] = fmaf(h[q], C.lds[i * N + q], y[q & 1]);
            }
          }
        }
        if constexpr (NW > 1) s_y[me.wave][i][threadIdx.x & 63] = y[0] + y[1];
        else z[i] *= y[0] + y[1];
        keep_live(z[i]);   // made here, not where it is stored: the states of all rows would have to wait for it
      }
    };
    const auto part = [&](int i, int k, const typename S::Raw& rb, const typename S::Raw& rc) {
      part_of(std::false_type{}, i, k, rb, rc);
    };
    const auto leave = [&] {   // after a sequence's last row
      if (p.st_out) {
        const int64_t k = at.row();
        if (k >= 0) me.store(p, p.st_out, k, h);
      }
      at.next();
    };
    if (tame && tb >= t0 && tb > at.beg && tb + TT <= at.end && tb + TT <= t1) {   // all of one sequence
      if (p.hs) me.store(p, p.hs, tb / TT, h);
      over_tile<1>(B, C, true, tb, part);
      if (tb + TT == at.end) leave();
    } else {
#pragma unroll
      for (int i = 0; i < TT; ++i) {
        const int t = tb + i;
        if (t < t0) continue;
        if (t >= t1) break;
        if (t == at.beg) {
          const int64_t k = p.st_in ? at.row() : -1;
          if (k >= 0) me.load(p, p.first && at.end > t1 ? p.first : p.st_in, p.first && at.end > t1 ? c : k, h);
          else zero(h);
          if (p.init) me.store(p, p.init, at.s, h);
        } else if (i == 0 && p.hs) {
          me.store(p, p.hs, tb / TT, h);
        }
#pragma unroll
        for (int k = 0; k < S::PARTS; ++k) part_of(std::bool_constant<PAD>{}, i, k, B.fetch(t, k), C.fetch(t, k));
        if (t + 1 == at.end) leave();
      }
    }
    if constexpr (NW > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TT; ++i) z[i] *= s_y[0][i][threadIdx.x & 63] + s_y[1][i][threadIdx.x & 63];
    }
    if (me.mine) {
#pragma unroll
      for (int i = 0; i < TT; ++i)
        if (i % NW == me.wave && tb + i >= t0 && tb + i < t1) put<T>((T*)p.y + (int64_t)(tb + i) * p.ldy + me.col0, me.col, z[i]);
    }
    if constexpr (!SC) __syncthreads();
  }
}

// ------------------------------------------------------------------ backward
//
// With e = dy silu(z): g_t = C_t e_t + a_(t+1) g_(t+1), the gradient of h_t; what a chunk hands to the one before
// it is r = a_t g_t at its first row, again a linear recurrence (k_scan_back_local, k_scan_carry).
// k_scan_back then goes over a chunk's tiles from the last to the first: each tile's states forwards from the
// forward's checkpoint, kept in registers half a tile at a time, then g backwards.

template <typename T, int N, int NW, bool SC>
__global__ __launch_bounds__(64 * NW) void k_scan_back_local(ScanP p, ScanG o) {
  __shared__ __align__(16) float s_C[NW * States<T, N, SC>::WORDS];
  const int c = blockIdx.x / p.nct, tile = blockIdx.x % p.nct;
  const Lane me(p, tile, N);
  const States<T, N, SC> C(p.C, p.ldC, p.n, me, s_C);
  const SeqRange r = seq_range(p.q);
  int t0, t1;
  chunk_rows(p, r, c, t0, t1);
  int flag = CARRY_NONE;
  SeqAt at{0, 0, 0};
  if (t0 < t1) {
    at = seq_find(p.q.off, r.n, t0);
    if (at.beg < t0) flag = at.end <= t1 ? CARRY_OWN : CARRY_ADD;
  }
  if (tile == 0 && threadIdx.x == 0) p.flag[c] = flag;
  if (flag == CARRY_NONE) return;
  const int stop = min(at.end, t1);
  float A2[N], g[N];
  me.decay(p, A2);
  zero(g);
  const float bias = p.bias ? p.bias[me.col0 + me.col] : 0.f;
  float sum = 0.f;
  for (int tb = t0 + (stop - 1 - t0) / TT * TT; tb >= t0; tb -= TT) {
    float u[TT], z[TT], e[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      const int row = min(tb + i, stop - 1);
      u[i] = me.at<T>(p.delta, p.ldd, row);
      z[i] = p.z ? me.at<T>(p.z, p.ldz, row) : 1.f;
      e[i] = me.at<float>(o.dy, o.lddy, row);
    }
    C.stage(tb, stop - 1);
    if constexpr (!SC) __syncthreads();
    step_sizes(p, bias, u);
    gates(p, z);
    using S = States<T, N, SC>;
    const auto part = [&](int i, int k, const typename S::Raw& rc, const typename S::Raw&) {
      const float dt = u[i], ee = e[i] * z[i];
      if (k == 0) sum += dt;
      float cc[S::M];
      C.values(rc, i, k, cc);
#pragma unroll
      for (int s = 0; s < S::M; ++s) {
        float& gs = g[k * S::M + s];
        gs = __builtin_amdgcn_exp2f(dt * A2[k * S::M + s]) * fmaf(ee, cc[s], gs);
      }
    };
    if (tb + TT <= stop) {
      over_tile<-1>(C, C, false, tb, part);
    } else {
#pragma unroll
      for (int i = TT - 1; i >= 0; --i) {
        if (tb + i >= stop) continue;
#pragma unroll
        for (int k = 0; k < S::PARTS; ++k) {
          const typename S::Raw rc = C.fetch(tb + i, k);
          part(i, k, rc, rc);
        }
      }
    }
    if constexpr (!SC) __syncthreads();
  }
  me.store(p, p.E, c, g);
  if (me.mine && me.wave == 0) p.sumdt[(int64_t)c * p.d + me.col0 + me.col] = sum;
}

// PAD: fewer than NP states; as in k_scan_out, but in all mixed tiles: 2 to 5% of a training call, 1 to 9% in every tile.
template <typename T, int SPL, int NB, bool PAD>
__global__ __launch_bounds__(64 * NB, 2) void k_scan_back(ScanP p, ScanG o) {
  using P = Place<SPL, NB>;
  constexpr int NP = P::NP, HT = TT / 2;
  __shared__ __align__(16) float s_dt[TT][CT], s_dx[TT][CT], s_e[TT][CT];
  __shared__ float s_x[TT][CT], s_s[TT][CT], s_z[TT][CT];     // x, d dt / d delta, dy silu'(z)
  __shared__ __align__(16) float s_B[TT * NP], s_C[TT * NP];
  __shared__ __align__(16) float s_bc[TT][4][2][NP];          // dB, dC of a tile, from each 16 lanes
  __shared__ float s_red[NB > 1 ? NB : 1][3][NB > 1 ? TT : 1][CT];
  __shared__ int s_tame[NB];
  const int c = blockIdx.x / p.nct, tile = blockIdx.x % p.nct;
  P me(p, tile);
  const SeqRange r = seq_range(p.q);
  int t0, t1;
  chunk_rows(p, r, c, t0, t1);
  if (t0 >= t1) return;
  SeqWalk at(p.q, r, t1 - 1);
  const float* init = *p.carried ? p.init : nullptr;
  float A2[4][SPL], f[4][SPL], dA[4][SPL];   // f: what flows from the row behind
  me.decay(p, A2);
  zero_state(&f[0][0], 4 * SPL);
  zero_state(&dA[0][0], 4 * SPL);
  if (p.nchunk > 1 && at.end > t1) me.load(p, p.E, c, f);
  const bool mine = me.lane < me.left;
  uint32_t col = mine ? me.lane : 0;
  const float bias = p.bias ? p.bias[me.ch0 + col] : 0.f, D = p.D ? p.D[me.ch0 + col] : 0.f;
  float dD = 0.f, db = 0.f;
  for (int tb = (t1 - 1) / TT * TT; tb + TT > t0; tb -= TT) {
    const int tlo = max(tb, t0), thi = min(tb + TT, t1);
    // addresses are formed in the tile, not kept over all of them (opaque)
    asm volatile("" : "+v"(me.lane), "+v"(col));
    me.cb = me.lane & ~3;
    me.n0 = me.wid * 4 * SPL + (me.lane & 3) * SPL;
    float* my_bc = &s_bc[0][me.lane >> 4][me.lane >> 2 & 1][me.n0];   // (two lanes write each value, the same)
    const bool is_C = me.lane & 4;
    float all = 0.f;   // not finite where a value of the tile is not
    {
      constexpr int U = (TT + NB - 1) / NB;
      float u[U], x[U], z[U], dy[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t row = min(max(tb + k * NB + me.wid, t0), t1 - 1);
        u[k] = Elem<T>::load((const T*)p.delta + row * p.ldd + me.ch0, col) + bias;
        x[k] = Elem<T>::load((const T*)p.x + row * p.ldx + me.ch0, col);
        z[k] = p.z ? Elem<T>::load((const T*)p.z + row * p.ldz + me.ch0, col) : 0.f;
        dy[k] = (o.dy + row * o.lddy + me.ch0)[col];
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int i = k * NB + me.wid;
        if (NB > 1 && i >= TT) break;
        float e = dy[k];
        if (p.z) {
          const float sg = sigmoid_hw(z[k]);
          e = dy[k] * (z[k] * sg);
          s_z[i][me.lane] = dy[k] * (sg * fmaf(z[k], 1.f - sg, 1.f));
        }
        const float dt = mine ? step_size(p, u[k]) : 0.f;
        s_x[i][me.lane] = x[k];
        s_s[i][me.lane] = p.softplus ? sigmoid_hw(u[k]) : 1.f;
        s_dt[i][me.lane] = dt;
        s_dx[i][me.lane] = mine ? dt * x[k] : 0.f;
        s_e[i][me.lane] = mine ? e : 0.f;
        if (PAD) all = fmaf(dt, x[k], all) + e;
      }
    }
    bool tame = !PAD || !__any(mine && !(fabsf(all) < INFINITY));
    if constexpr (PAD && NB > 1) s_tame[me.wid] = tame;
    stage_states<T, NP, 64 * NB>(p.B, p.ldB, p.n, me.g * p.n, tb, t1 - 1, s_B);
    stage_states<T, NP, 64 * NB>(p.C, p.ldC, p.n, me.g * p.n, tb, t1 - 1, s_C);
    __syncthreads();
    if constexpr (PAD && NB > 1) {
#pragma unroll
      for (int w = 0; w < NB; ++w) tame = tame && __builtin_amdgcn_readfirstlane(s_tame[w]);
    }
    while (at.beg > tlo) at.prev();
    // what a row's channel gets (lane l: channel l) once its sums over the states are complete
    const auto finish = [&](int i, float y, float sx, float su) {
      const int64_t t = tb + i;
      const float x = s_x[i][me.lane], e = s_e[i][me.lane];
      const float du = fmaf(sx, x, su * LN2) * s_s[i][me.lane];
      if (mine) {
        const float dxr = sx * s_dt[i][me.lane];
        (o.dx + t * o.lddx + me.ch0)[col] = p.D ? fmaf(D, e, dxr) : dxr;
        (o.ddelta + t * o.lddd + me.ch0)[col] = du;
        if (p.z) (o.dz + t * o.lddz + me.ch0)[col] = s_z[i][me.lane] * (p.D ? fmaf(D, x, y) : y);
      }
      dD = fmaf(e, x, dD);
      db += du;
    };
    // Half a tile: the states that enter its rows (hb), forwards from the checkpoint, then its rows backwards.  Eight
    // rows' states would be 128 registers and leave one wave a SIMD; so the first half's rows are gone over twice.
    const auto half = [&](auto first_row, auto one_sequence) {
      constexpr int I0 = decltype(first_row)::value;
      constexpr bool ONE = decltype(one_sequence)::value;
      const auto real = [&](int s, float v) { return !PAD || ONE || me.n0 + s < p.n ? v : 0.f; };
      float hb[HT][4][SPL];
      {
        float h[4][SPL];
        zero_state(&h[0][0], 4 * SPL);
        if (ONE || at.beg < tlo) me.load(p, p.hs, tb / TT, h);
#pragma unroll
        for (int i = 0; i < I0 + HT; ++i) {
          const int t = tb + i;
          if (!ONE && t >= tlo && t < thi) {
            if (t == at.end) at.next();
            if (t == at.beg) {
              if (init && at.row() >= 0) me.load(p, init, at.s, h);
              else zero_state(&h[0][0], 4 * SPL);
            }
          }
          if (i >= I0) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int s = 0; s < SPL; ++s) hb[i - I0 < 0 ? 0 : i - I0][k][s] = h[k][s];
          }
          if (i + 1 < I0 + HT) {
            float dt[4], dx[4], b[SPL];
            lds_get<4>(&s_dt[i][me.cb], dt);
            lds_get<4>(&s_dx[i][me.cb], dx);
            lds_get<SPL>(&s_B[i * NP + me.n0], b);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int s = 0; s < SPL; ++s)
                h[k][s] = real(s, fmaf(__builtin_amdgcn_exp2f(dt[k] * A2[k][s]), h[k][s], dx[k] * b[s]));
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      // the decays and inputs are formed again below: kept from above they would be hundreds of registers
      asm volatile("" ::: "memory");
      float yv[HT], gx[HT], gu[HT];
#pragma unroll
      for (int j = HT - 1; j >= 0; --j) {
        const int i = I0 + j, t = tb + i;
        yv[j] = gx[j] = gu[j] = 0.f;
        if (!ONE) {
          if (t < tlo || t >= thi) continue;
          while (at.beg > t) at.prev();
          if (t + 1 == at.end) zero_state(&f[0][0], 4 * SPL);
        }
        float dt[4], dx[4], e[4], b[SPL], cc[SPL], y4[4], x4[4], u4[4], vB[SPL], vC[SPL];
        lds_get<4>(&s_dt[i][me.cb], dt);
        lds_get<4>(&s_dx[i][me.cb], dx);
        lds_get<4>(&s_e[i][me.cb], e);
        lds_get<SPL>(&s_B[i * NP + me.n0], b);
        lds_get<SPL>(&s_C[i * NP + me.n0], cc);
#pragma unroll
        for (int s = 0; s < SPL; ++s) vB[s] = vC[s] = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          y4[k] = x4[k] = u4[k] = 0.f;
#pragma unroll
          for (int s = 0; s < SPL; ++s) {
            const float a = __builtin_amdgcn_exp2f(dt[k] * A2[k][s]);
            const float h = ONE && j + 1 < HT ? hb[j + 1 < HT ? j + 1 : j][k][s] : real(s, fmaf(a, hb[j][k][s], dx[k] * b[s]));
            const float g = real(s, fmaf(e[k], cc[s], f[k][s]));
            f[k][s] = real(s, a * g);
            const float w = f[k][s] * hb[j][k][s];
            y4[k] = fmaf(h, cc[s], y4[k]);
            x4[k] = fmaf(g, b[s], x4[k]);
            u4[k] = fmaf(w, A2[k][s], u4[k]);
            dA[k][s] = fmaf(w, dt[k], dA[k][s]);
            vB[s] = fmaf(g, dx[k], vB[s]);
            vC[s] = fmaf(h, e[k], vC[s]);
          }
        }
        yv[j] = quad_sums(y4);
        gx[j] = quad_sums(x4);
        gu[j] = quad_sums(u4);
        if constexpr (NB > 1) {
          s_red[me.wid][0][i][me.lane] = yv[j];
          s_red[me.wid][1][i][me.lane] = gx[j];
          s_red[me.wid][2][i][me.lane] = gu[j];
        } else {
          keep_live(yv[j]);
          keep_live(gx[j]);
          keep_live(gu[j]);
        }
        float v[SPL];
#pragma unroll
        for (int s = 0; s < SPL; ++s) {
          vB[s] += dpp<ROW_ROR4>(vB[s]);
          vC[s] += dpp<ROW_ROR4>(vC[s]);
          vB[s] += dpp<ROW_ROR8>(vB[s]);
          vC[s] += dpp<ROW_ROR8>(vC[s]);
          v[s] = is_C ? vC[s] : vB[s];
        }
        lds_put<SPL>(my_bc + i * 8 * NP, v);
#pragma unroll
        for (int k = 0; k < 4; ++k)   // added now, not at the end of the rows with all their terms kept
#pragma unroll
          for (int s = 0; s < SPL; ++s) keep_live(dA[k][s]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (NB == 1) {
#pragma unroll
        for (int j = HT - 1; j >= 0; --j)
          if (ONE || (tb + I0 + j >= tlo && tb + I0 + j < thi)) finish(I0 + j, yv[j], gx[j], gu[j]);
      }
    };
    const auto both = [&](auto one) {
      half(std::integral_constant<int, HT>{}, one);
      if (!decltype(one)::value) {
        while (at.beg > tlo) at.prev();
      }
      half(std::integral_constant<int, 0>{}, one);
    };
    if (tame && at.beg < tb && tlo == tb && thi == tb + TT && tb + TT <= at.end) {   // all of one sequence
      if (tb + TT == at.end) zero_state(&f[0][0], 4 * SPL);
      both(std::true_type{});
    } else {
      both(std::false_type{});
    }
    __syncthreads();
#pragma unroll 1
    for (int e = threadIdx.x; e < TT * 2 * NP; e += 64 * NB) {
      const int i = e / (2 * NP), w = e / NP & 1, s = e % NP, t = tb + i;
      if (t < tlo || t >= thi || s >= p.n) continue;
      const float v = (s_bc[i][0][w][s] + s_bc[i][1][w][s]) + (s_bc[i][2][w][s] + s_bc[i][3][w][s]);
      if (p.tpg > 1) o.bc[(((int64_t)tile * p.q.max_rows + t) * 2 + w) * p.n + s] = v;
      else if (w == 0) o.dB[(int64_t)t * o.lddB + me.g * p.n + s] = v;
      else o.dC[(int64_t)t * o.lddC + me.g * p.n + s] = v;
    }
    if constexpr (NB > 1) {
      for (int i = me.wid; i < TT; i += NB) {
        if (tb + i < tlo || tb + i >= thi) continue;
        float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NB; ++w)
#pragma unroll
          for (int k = 0; k < 3; ++k) v[k] += s_red[w][k][i][me.lane];
        finish(i, v[0], v[1], v[2]);
      }
    }
    __syncthreads();
  }
  float* part = o.part + (int64_t)c * (p.n + 2) * p.d;
  me.store(p, part, 0, dA);
  if constexpr (NB > 1) {
    s_dt[me.wid][me.lane] = dD;
    s_dx[me.wid][me.lane] = db;
    __syncthreads();
    dD = db = 0.f;
    for (int w = 0; w < NB; ++w) {
      dD += s_dt[w][me.lane];
      db += s_dx[w][me.lane];
    }
  }
  if (me.wid == 0 && mine) {
    (part + (int64_t)p.n * p.d + me.ch0)[col] = dD;
    (part + (int64_t)(p.n + 1) * p.d + me.ch0)[col] = db;
  }
}

// dB, dC from the tiles' shares: a thread per row, operand, group and state.
__global__ __launch_bounds__(256) void k_scan_sum_bc(ScanP p, ScanG o) {
  const SeqRange r = seq_range(p.q);
  const int gn = p.groups * p.n;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = e / (2 * gn);
  if (t < r.lo || t >= r.hi) return;
  const int w = (int)(e / gn & 1), j = (int)(e % gn), g = j / p.n, s = j % p.n;
  float v = 0.f;
  for (int k = 0; k < p.tpg; ++k) v += o.bc[(((int64_t)(g * p.tpg + k) * p.q.max_rows + t) * 2 + w) * p.n + s];
  if (w == 0) o.dB[t * o.lddB + j] = v;
  else o.dC[t * o.lddC + j] = v;
}

// ------------------------------------------------------------------ single rows

// A thread per row and V neighbouring channels.  Its states are n reads and writes a row of the table apart (a
// wave's are 1 KB together for V = 4), eight of them in flight; that traffic bounds it: 16,000 rows x 256 channels x 16
// states in 119 us, 4.7 TB/s, what a large copy reaches.  Few rows: the launch (400 x 32: 5.5 us).
template <int V>
__device__ __forceinline__ void get_f(const float* p, float (&v)[V]) {
  if constexpr (V == 4) {
    const float4 f = *(const float4*)p;
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
    v[0] = p[0];
  }
}
template <typename T, int V>
__global__ __launch_bounds__(256) void k_scan_step(ScanP p, const int32_t* n_rows, int64_t max_rows) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int dv = p.d / V;
  const int64_t row = e / dv;
  if (row >= eff_count(max_rows, n_rows)) return;
  const int ch = (int)(e % dv) * V, g = ch / p.per;
  const int64_t k = seq_slot(p.q.slot, p.q.n_slots, row);
  const T *B = (const T*)p.B + row * p.ldB + g * p.n, *C = (const T*)p.C + row * p.ldC + g * p.n;
  const float* in = p.st_in && k >= 0 ? p.st_in + k * p.n * p.d + ch : nullptr;
  float* out = p.st_out && k >= 0 ? p.st_out + k * p.n * p.d + ch : nullptr;
  float x[V], z[V], dt[V], y[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float u = Elem<T>::load((const T*)p.delta, row * p.ldd + ch + v) + (p.bias ? p.bias[ch + v] : 0.f);
    x[v] = Elem<T>::load((const T*)p.x, row * p.ldx + ch + v);
    z[v] = p.z ? Elem<T>::load((const T*)p.z, row * p.ldz + ch + v) : 0.f;
    dt[v] = step_size(p, u);
    y[v] = 0.f;
  }
  constexpr int G = 8;
  for (int i0 = 0; i0 < p.n; i0 += G) {
    float h[G][V], A[G][V], b[G], c[G];
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int64_t s = min(i0 + i, p.n - 1);
#pragma unroll
      for (int v = 0; v < V; ++v) h[i][v] = 0.f;
      if (in) get_f<V>(in + s * p.d, h[i]);
      get_f<V>(p.A + s * p.d + ch, A[i]);
      b[i] = Elem<T>::load(B, s);
      c[i] = Elem<T>::load(C, s);
    }
#pragma unroll
    for (int i = 0; i < G; ++i) {
      if (i0 + i >= p.n) break;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[i][v] = fmaf(__builtin_amdgcn_exp2f(dt[v] * (A[i][v] * LOG2E)), h[i][v], dt[v] * x[v] * b[i]);
        y[v] = fmaf(h[i][v], c[i], y[v]);
      }
      if (out) {
        float* o = out + (int64_t)(i0 + i) * p.d;
        if constexpr (V == 4) *(float4*)o = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
        else o[0] = h[i][0];
      }
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (p.D) y[v] = fmaf(p.D[ch + v], x[v], y[v]);
    if (p.z) y[v] *= silu_(z[v]);
    Elem<T>::store((T*)p.y, row * p.ldy + ch + v, y[v]);
  }
}

// ------------------------------------------------------------------ host

int scan_tiles(const mtgnn_scan_dims* d) { return d->groups * (int)cdiv(d->d / d->groups, CT); }

// Rows of a chunk (a multiple of TT): enough chunks for `waves` waves.  With 2,048, 4,096 and 8,192 of them (us):
// forward of 32,768 x 2,048 local 274, 234, 223, out 602, 370, 383, carry 30 (64 runs), 13, 22; backward of 16,384 x 1,024
// local 121, 84, 88, k_scan_back 344, 352, 365, sums 6, 10, 17.
int scan_chunk(const mtgnn_scan_dims* d, int64_t rows, int64_t waves) {
  const int64_t blocks = std::max<int64_t>(1, waves / (scan_tiles(d) * cdiv(d->n, 16)));
  const int64_t ch = cdiv(cdiv(std::max<int64_t>(rows, 1), blocks), TT) * TT;
  return (int)std::min<int64_t>(ch, int64_t(1) << 30);
}
constexpr int64_t FWD_WAVES = 4096, BWD_WAVES = 4096;

size_t al(size_t b) { return (b + 255) & ~size_t(255); }

ScanP scan_params(const mtgnn_seqs* q, const mtgnn_scan_inputs* in, const mtgnn_scan_dims* d) {
  ScanP p{};
  if (q) p.q = seqs_of(q);
  p.x = in->x; p.delta = in->delta; p.B = in->B; p.C = in->C; p.z = in->z;
  p.ldx = in->ldx; p.ldd = in->lddelta; p.ldB = in->ldB; p.ldC = in->ldC; p.ldz = in->ldz;
  p.A = in->A; p.D = in->D; p.bias = in->delta_bias;
  p.d = d->d; p.n = d->n; p.groups = d->groups; p.per = d->d / d->groups;
  p.tpg = (int)cdiv(p.per, CT); p.nct = d->groups * p.tpg; p.softplus = d->softplus;
  return p;
}
// Every state row's groups of four channels that a thread takes are 16-byte aligned.
int scan_vec(const ScanP& p, const void* a, const void* b) {
  return p.d % 4 == 0 && p.per % 4 == 0 && ((uintptr_t)a | (uintptr_t)b | (uintptr_t)p.A) % 16 == 0;
}

struct ScanWs {
  size_t E, sumdt, flag, first, part, bc, total;
};
ScanWs scan_ws_layout(const mtgnn_scan_dims* d, int64_t rows, bool back) {
  const int64_t nchunk = cdiv(std::max<int64_t>(rows, 1), scan_chunk(d, rows, back ? BWD_WAVES : FWD_WAVES));
  const size_t nd = (size_t)d->n * d->d;
  ScanWs w{};
  size_t o = 0;
  w.E = o; o += al(nchunk * nd * 4);
  w.sumdt = o; o += al(nchunk * (size_t)d->d * 4);
  w.flag = o; o += al(nchunk * 4);
  w.first = o; if (!back) o += al(nchunk * nd * 4);
  w.part = o; if (back) o += al(nchunk * (nd + 2 * (size_t)d->d) * 4);
  w.bc = o;
  const int nct = scan_tiles(d);
  if (back && nct > d->groups) o += al((size_t)nct * rows * 2 * d->n * 4);
  w.total = o;
  return w;
}

template <typename F>
void scan_variant(int dtype, int n, F f) {
  const auto by = [&](auto t) {
    using T = decltype(t);
    if (n <= 4) f.template operator()<T, 1, 1>();
    else if (n <= 8) f.template operator()<T, 2, 1>();
    else if (n <= 16) f.template operator()<T, 4, 1>();
    else if (n <= 32) f.template operator()<T, 4, 2>();
    else if (n <= 48) f.template operator()<T, 4, 3>();
    else f.template operator()<T, 4, 4>();
  };
  if (dtype == MTGNN_BF16) by(uint16_t{});
  else by(float{});
}

// The lane-per-channel kernels: n rounded up, and whether B and C come by scalar loads: their rows are whole words (n of
// a supported number), and sequences of a tile's rows or more leave most tiles inside one, where the next words are
// requested ahead.  k_scan_out and k_scan_local by scalar loads against LDS: 370 and 234 us against 540 and 231
// (5 sequences, 32,768 rows x 2,048, bfloat16); 31.5 and 15.2 against 28.5 and 14.0 (6,000 sequences of 8,000 rows x 100).
template <typename F>
void scan_lane_variant(const ScanP& p, int dtype, F f) {
  const int N = p.n <= 4 ? 4 : p.n <= 8 ? 8 : p.n <= 16 ? 16 : p.n <= 32 ? 32 : 64;   // 64: two waves of 32
  const bool words = p.n == N && p.q.max_rows >= TT * p.q.max_seq &&
                     (dtype == MTGNN_F32 || (p.ldB % 2 == 0 && p.ldC % 2 == 0 && (uintptr_t)p.B % 4 == 0 &&
                                            (uintptr_t)p.C % 4 == 0));
  const auto by = [&](auto t) {
    using T = decltype(t);
    const auto with = [&](auto sc) {
      constexpr bool SC = decltype(sc)::value;
      if (N == 4) f.template operator()<T, 4, 1, SC>();
      else if (N == 8) f.template operator()<T, 8, 1, SC>();
      else if (N == 16) f.template operator()<T, 16, 1, SC>();
      else if (N == 32) f.template operator()<T, 32, 1, SC>();
      else f.template operator()<T, 32, 2, SC>();
    };
    if (words) with(std::true_type{});
    else with(std::false_type{});
  };
  if (dtype == MTGNN_BF16) by(uint16_t{});
  else by(float{});
}

struct LaunchLocal {
  const ScanP& p;
  unsigned grid;
  hipStream_t s;
  template <typename T, int N, int NW, bool SC> void operator()() const { k_scan_local<T, N, NW, SC><<<grid, 64 * NW, 0, s>>>(p); }
};
struct LaunchOut {
  const ScanP& p;
  unsigned grid;
  hipStream_t s;
  template <typename T, int N, int NW, bool SC> void operator()() const {
    if constexpr (!SC) {
      if (p.n < N * NW) return k_scan_out<T, N, NW, false, true><<<grid, 64 * NW, 0, s>>>(p);
    }
    k_scan_out<T, N, NW, SC, false><<<grid, 64 * NW, 0, s>>>(p);
  }
};
struct LaunchBackLocal {
  const ScanP& p;
  const ScanG& g;
  unsigned grid;
  hipStream_t s;
  template <typename T, int N, int NW, bool SC> void operator()() const {
    k_scan_back_local<T, N, NW, SC><<<grid, 64 * NW, 0, s>>>(p, g);
  }
};
struct LaunchBack {
  const ScanP& p;
  const ScanG& g;
  unsigned grid;
  hipStream_t s;
  template <typename T, int SPL, int NB> void operator()() const {
    if (p.n < 4 * SPL * NB) k_scan_back<T, SPL, NB, true><<<grid, 64 * NB, 0, s>>>(p, g);
    else k_scan_back<T, SPL, NB, false><<<grid, 64 * NB, 0, s>>>(p, g);
  }
};

}  // namespace

size_t scan_ws(const mtgnn_scan_dims* d, int64_t rows, bool back) { return scan_ws_layout(d, rows, back).total; }

// Saved: a flag (whether there are first states), the checkpoints, the first states.
size_t scan_save(const mtgnn_scan_dims* d, int64_t rows, int64_t max_seq, bool carried) {
  const size_t nd = (size_t)d->n * d->d * 4;
  return 256 + al(cdiv(std::max<int64_t>(rows, 1), TT) * nd) + (carried ? al(max_seq * nd) : 0);
}
static void scan_save_at(ScanP& p, const mtgnn_scan_dims* d, int64_t rows, void* save) {
  char* b = (char*)save;
  p.carried = (int32_t*)b;
  p.hs = (float*)(b + 256);
  p.init = (float*)(b + 256 + al(cdiv(std::max<int64_t>(rows, 1), TT) * ((size_t)d->n * d->d * 4)));
}

static mtgnn_status scan_carry(const ScanP& p, int back, hipStream_t s) {
  const int64_t nd = (int64_t)p.n * p.d;
  if (p.nchunk > 256) k_scan_carry<64><<<(unsigned)cdiv(nd, 16), 1024, 0, s>>>(p, back);
  else k_scan_carry<16><<<(unsigned)cdiv(nd, 64), 1024, 0, s>>>(p, back);
  MTGNN_CHECK_LAUNCH("scan_carry");
  return MTGNN_OK;
}

mtgnn_status scan_impl(const mtgnn_seqs* q, const mtgnn_scan_inputs* in, const mtgnn_scan_dims* d,
                       const float* state_in, float* state_out, void* y, int64_t ldy, void* save, void* ws,
                       hipStream_t s) {
  ScanP p = scan_params(q, in, d);
  const int64_t rows = q->max_rows;
  p.ch = scan_chunk(d, rows, FWD_WAVES);
  p.nchunk = (int)cdiv(rows, p.ch);
  p.st_in = state_in; p.st_out = state_out; p.y = y; p.ldy = ldy;
  if (save) {
    scan_save_at(p, d, rows, save);
    if (!state_in) p.init = nullptr;
  }
  const ScanWs w = scan_ws_layout(d, rows, false);
  p.E = (float*)((char*)ws + w.E);
  p.sumdt = (float*)((char*)ws + w.sumdt);
  p.flag = (int32_t*)((char*)ws + w.flag);
  if (state_in && state_in == state_out && p.nchunk > 1) p.first = (float*)((char*)ws + w.first);
  const unsigned grid = (unsigned)((int64_t)p.nchunk * p.nct);
  if (p.nchunk > 1) {
    scan_lane_variant(p, d->dtype, LaunchLocal{p, grid, s});
    MTGNN_CHECK_LAUNCH("scan_local");
    MTGNN_TRY(scan_carry(p, 0, s));
  }
  scan_lane_variant(p, d->dtype, LaunchOut{p, grid, s});
  MTGNN_CHECK_LAUNCH("scan_out");
  return MTGNN_OK;
}

mtgnn_status scan_bwd_impl(const mtgnn_seqs* q, const float* dy, int64_t lddy, const mtgnn_scan_inputs* in,
                           const mtgnn_scan_dims* d, const void* save, const mtgnn_scan_grads* g, void* ws,
                           hipStream_t s) {
  ScanP p = scan_params(q, in, d);
  const int64_t rows = q->max_rows;
  p.ch = scan_chunk(d, rows, BWD_WAVES);
  p.nchunk = (int)cdiv(rows, p.ch);
  p.vec = scan_vec(p, ws, save);
  scan_save_at(p, d, rows, const_cast<void*>(save));
  const ScanWs w = scan_ws_layout(d, rows, true);
  p.E = (float*)((char*)ws + w.E);
  p.sumdt = (float*)((char*)ws + w.sumdt);
  p.flag = (int32_t*)((char*)ws + w.flag);
  ScanG o{};
  o.dy = dy; o.lddy = lddy;
  o.dx = g->dx; o.ddelta = g->ddelta; o.dB = g->dB; o.dC = g->dC; o.dz = g->dz;
  o.lddx = g->lddx; o.lddd = g->ldddelta; o.lddB = g->lddB; o.lddC = g->lddC; o.lddz = g->lddz;
  o.part = (float*)((char*)ws + w.part);
  o.bc = (float*)((char*)ws + w.bc);
  const unsigned grid = (unsigned)((int64_t)p.nchunk * p.nct);
  if (p.nchunk > 1) {
    scan_lane_variant(p, d->dtype, LaunchBackLocal{p, o, grid, s});
    MTGNN_CHECK_LAUNCH("scan_back_local");
    MTGNN_TRY(scan_carry(p, 1, s));
  }
  scan_variant(d->dtype, d->n, LaunchBack{p, o, grid, s});
  MTGNN_CHECK_LAUNCH("scan_back");
  if (p.tpg > 1) {
    k_scan_sum_bc<<<(unsigned)cdiv(rows * 2 * d->groups * d->n, 256), 256, 0, s>>>(p, o);
    MTGNN_CHECK_LAUNCH("scan_sum_bc");
  }
  const int64_t nd = (int64_t)d->n * d->d;
  k_sum_parts<<<(unsigned)cdiv(nd + 2 * d->d, 16), 256, 0, s>>>(p.q, p.ch, 0, o.part, nd + 2 * d->d, nd, g->dA, d->d,
                                                                g->dD, g->ddelta_bias);
  MTGNN_CHECK_LAUNCH("scan_sum_parts");
  return MTGNN_OK;
}

mtgnn_status scan_step_impl(const int32_t* slot, const int32_t* n_rows, int64_t max_rows, int64_t n_slots,
                            const mtgnn_scan_inputs* in, const mtgnn_scan_dims* d, const float* state_in,
                            float* state_out, void* y, int64_t ldy, hipStream_t s) {
  ScanP p = scan_params(nullptr, in, d);
  p.q.slot = slot;
  p.q.n_slots = n_slots;
  p.st_in = state_in; p.st_out = state_out; p.y = y; p.ldy = ldy;
  // Four channels a thread where that leaves four blocks a CU: 119 against 122 us (16,000 rows x 256); with few rows one
  // channel a thread has the more loads in flight: 5.5 against 7.3 us (400 x 32).
  const bool four = max_rows * d->d >= (int64_t(1) << 20) && scan_vec(p, state_in, state_out);
  const unsigned grid = (unsigned)cdiv(max_rows * (d->d / (four ? 4 : 1)), 256);
  const auto launch = [&](auto t) {
    using T = decltype(t);
    if (four) k_scan_step<T, 4><<<grid, 256, 0, s>>>(p, n_rows, max_rows);
    else k_scan_step<T, 1><<<grid, 256, 0, s>>>(p, n_rows, max_rows);
  };
  if (d->dtype == MTGNN_BF16) launch(uint16_t{});
  else launch(float{});
  MTGNN_CHECK_LAUNCH("scan_step");
  return MTGNN_OK;
}

}  // namespace mtgnn
