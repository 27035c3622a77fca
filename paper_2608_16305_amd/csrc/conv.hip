// Short causal convolution over ragged sequences, channel by channel: whole sequences, their backward, single rows.
//
//   y_t = act(b + sum_j w[j] x_(t - W + 1 + j))
//
// A lane holds V channels and a wave walks its chunk of rows a tile of eight at a time: the tile's rows and the
// W - 1 before it are requested together, and a row is read again only as another tile's margin (11 reads for 8, from
// the caches).  Where a sequence starts, its first W - 1 rows take the values that are missing from its slot's
// state instead of from the rows above.  Reading and writing the rows bounds it: 32,768 rows x 2,048 in bfloat16 take
// 80 us forward (3.4 TB/s) and 164 us backward (4.1 TB/s: x, dy in, dx out); 4,000 single rows 28 us with their
// states in the caches, 38 without.  8,000 rows x 100 of 6,000 sequences take 9 us, a chain of dependent reads (count, search,
// offsets, rows, state) in one wave a SIMD, and 4 us for the new states.
#include <algorithm>
#include <initializer_list>

#include "bf16_split.h"
#include "ops.h"
#include "seq.h"

namespace mtgnn {

namespace {

constexpr int TR = 8;   // rows of a tile

struct ConvP {
  Seqs q;
  const void *x, *w;
  const float* b;
  int64_t ldx, ldy;
  int d, act, ch;            // ch: rows of a wave's chunk
  int tiles;                 // blocks over the channels
  const void* st_in;         // forward: state table; backward: first states by sequence
  void *st_out, *save, *y;
  const float* dy;
  int64_t lddy, lddx;
  float *dx, *part;          // part: [chunk][W + 1][d]
};

template <typename T, int V>
__device__ __forceinline__ void get(const void* p, int64_t i, float (&v)[V]) {
  if constexpr (V == 4 && sizeof(T) == 2) {
    const uint2 u = *(const uint2*)((const T*)p + i);
    v[0] = lo_bf16(u.x); v[1] = hi_bf16(u.x); v[2] = lo_bf16(u.y); v[3] = hi_bf16(u.y);
  } else if constexpr (V == 4) {
    const float4 f = *(const float4*)((const T*)p + i);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else if constexpr (V == 2 && sizeof(T) == 2) {
    const uint32_t u = *(const uint32_t*)((const T*)p + i);
    v[0] = __uint_as_float(u << 16);
    v[1] = __uint_as_float(u & 0xffff0000u);
  } else if constexpr (V == 2) {
    const float2 f = *(const float2*)((const T*)p + i);
    v[0] = f.x;
    v[1] = f.y;
  } else {
    v[0] = Elem<T>::load((const T*)p, i);
  }
}
template <typename T, int V>
__device__ __forceinline__ void put(void* p, int64_t i, const float (&v)[V]) {
  if constexpr (V == 4 && sizeof(T) == 2) {
    *(uint2*)((T*)p + i) = make_uint2(cvt2_bf16(v[0], v[1]), cvt2_bf16(v[2], v[3]));
  } else if constexpr (V == 4) {
    *(float4*)((T*)p + i) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (V == 2 && sizeof(T) == 2) {
    *(uint32_t*)((T*)p + i) = cvt2_bf16(v[0], v[1]);
  } else if constexpr (V == 2) {
    *(float2*)((T*)p + i) = make_float2(v[0], v[1]);
  } else {
    Elem<T>::store((T*)p, i, v[0]);
  }
}

// Chunk and channels of this wave (four chunks a block).
template <int V>
struct Here {
  int chunk, col;
  bool mine;
  int t0, t1;
  __device__ __forceinline__ Here(const ConvP& p, const SeqRange& r) {
    const int tile = blockIdx.x % p.tiles;
    chunk = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / p.tiles) * 4 + (int)(threadIdx.x >> 6));
    col = (tile * 64 + (threadIdx.x & 63)) * V;
    mine = col < p.d;
    if (!mine) col = 0;
    const int64_t a = (int64_t)chunk * p.ch;
    t0 = (int)(a > r.lo ? a : r.lo);
    t1 = (int)(a + p.ch < r.hi ? a + p.ch : r.hi);
  }
};

// Of rows tb .. tb + N - 1 (those below hi): the place in its sequence and the row of the state table (or -1), with
// the walk moved to row tb + N.
template <int N, bool BY_SEQ>
__device__ __forceinline__ void places(SeqWalk& at, int tb, int t0, int hi, int (&pos)[N], int64_t (&st)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = tb + i;
    pos[i] = 0;
    st[i] = -1;
    if (t < t0 || t >= hi) continue;
    while (t >= at.end && at.s + 1 < at.n) at.next();
    pos[i] = t - at.beg;
    st[i] = at.row();
    if (BY_SEQ && st[i] >= 0) st[i] = at.s;
  }
}

// The W inputs of row i of a tile whose rows start W - 1 before it in xr: rows above, or of the first states.
template <int W, int V, int NX>
__device__ __forceinline__ void window(const float (&xr)[NX][V], const float (&sv)[W - 1][V], int i, int pos,
                                       float (&win)[W][V]) {
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int v = 0; v < V; ++v) win[j][v] = j < W - 1 && pos < W - 1 - j ? sv[j < W - 1 ? j : 0][v] : xr[i + j][v];
}
// The states that row i needs: sv[j] = state[pos + j] for j < W - 1 - pos.
template <typename T, int W, int V>
__device__ __forceinline__ void first_states(const ConvP& p, int pos, int64_t st, int col, float (&sv)[W - 1][V]) {
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
#pragma unroll
    for (int v = 0; v < V; ++v) sv[j][v] = 0.f;
    if (p.st_in && st >= 0 && pos < W - 1 - j) get<T, V>(p.st_in, (st * (W - 1) + pos + j) * p.d + col, sv[j]);
  }
}

template <typename T, int W, int V>
__global__ __launch_bounds__(256) void k_conv(ConvP p) {
  const SeqRange r = seq_range(p.q);
  const Here<V> me(p, r);
  if (me.t0 >= me.t1) return;
  SeqWalk at(p.q, r, me.t0);
  float w[W][V], b[V];
#pragma unroll
  for (int j = 0; j < W; ++j) get<T, V>(p.w, (int64_t)j * p.d + me.col, w[j]);
#pragma unroll
  for (int v = 0; v < V; ++v) b[v] = p.b ? p.b[me.col + v] : 0.f;
  const auto tile = [&](int tb, auto inside) {
    constexpr bool INSIDE = decltype(inside)::value;
    float xr[TR + W - 1][V], sv[INSIDE ? 1 : TR][W - 1][V];
#pragma unroll
    for (int i = 0; i < TR + W - 1; ++i)
      get<T, V>(p.x, (int64_t)min(max(tb + i - (W - 1), r.lo), me.t1 - 1) * p.ldx + me.col, xr[i]);
    int pos[TR];
    int64_t st[TR];
    if constexpr (!INSIDE) {
      places<TR, false>(at, tb, me.t0, me.t1, pos, st);
#pragma unroll
      for (int i = 0; i < TR; ++i) first_states<T, W, V>(p, pos[i], tb + i < me.t1 ? st[i] : -1, me.col, sv[i]);
    }
#pragma unroll
    for (int i = 0; i < TR; ++i) {
      if (tb + i >= me.t1) break;
      float win[W][V], y[V];
      window<W, V>(xr, sv[INSIDE ? 0 : i], i, INSIDE ? W : pos[i], win);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float a = b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) a = fmaf(w[j][v], win[j][v], a);
        y[v] = p.act ? silu_(a) : a;
      }
      if (me.mine) put<T, V>(p.y, (int64_t)(tb + i) * p.ldy + me.col, y);
    }
  };
  for (int tb = me.t0; tb < me.t1; tb += TR) {
    while (tb >= at.end && at.s + 1 < at.n) at.next();
    if (tb - at.beg >= W - 1 && tb + TR <= at.end) tile(tb, std::true_type{});
    else tile(tb, std::false_type{});
  }
}

// The states that a call leaves, and the ones it started from into save.  A thread per sequence and channel
// reads its old state before it writes, so the tables may be one.
template <typename T, int W>
__global__ __launch_bounds__(256) void k_conv_state(ConvP p) {
  const SeqRange r = seq_range(p.q);
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t s = e / p.d;
  if (s >= r.n) return;
  const int ch = (int)(e % p.d), beg = max(p.q.off[s], r.lo), len = min(p.q.off[s + 1], r.hi) - beg;
  if (len <= 0) return;
  const int64_t k = seq_slot(p.q.slot, p.q.n_slots, s);
  if (k < 0) return;
  T old[W - 1];
#pragma unroll
  for (int j = 0; j < W - 1; ++j)
    old[j] = p.st_in ? ((const T*)p.st_in)[(k * (W - 1) + j) * p.d + ch] : T(0);
  if (p.save) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) ((T*)p.save)[(s * (W - 1) + j) * p.d + ch] = old[j];
  }
  if (!p.st_out) return;
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int i = len - (W - 1) + j;   // row of the sequence that becomes entry j; before its first: an old entry
    T v = T(0);
    if (i >= 0) v = ((const T*)p.x)[(int64_t)(beg + i) * p.ldx + ch];
#pragma unroll
    for (int o = 0; o < W - 1; ++o)
      if (o == W - 1 + i) v = old[o];
    ((T*)p.st_out)[(k * (W - 1) + j) * p.d + ch] = v;
  }
}

// Backward.  A tile's slopes g = dy act'(pre) are formed for its eight rows and the W - 1 behind them, which it
// needs for its rows' dx; row t + k belongs to row t's sequence where its place in its own is k or more.  dw and db are
// summed over the chunk in registers, then over the chunks (k_sum_parts).
template <typename T, int W, int V>
__global__ __launch_bounds__(256) void k_conv_back(ConvP p) {
  constexpr int N = TR + W - 1;   // rows whose slopes are formed
  const SeqRange r = seq_range(p.q);
  const Here<V> me(p, r);
  if (me.t0 >= me.t1) return;
  SeqWalk at(p.q, r, me.t0);
  float w[W][V], b[V], dw[W][V], db[V];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    get<T, V>(p.w, (int64_t)j * p.d + me.col, w[j]);
#pragma unroll
    for (int v = 0; v < V; ++v) dw[j][v] = 0.f;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    b[v] = p.b ? p.b[me.col + v] : 0.f;
    db[v] = 0.f;
  }
  const auto tile = [&](int tb, auto inside) {
    constexpr bool INSIDE = decltype(inside)::value;
    float xr[N + W - 1][V], g[N][V], sv[INSIDE ? 1 : N][W - 1][V];
#pragma unroll
    for (int i = 0; i < N + W - 1; ++i)
      get<T, V>(p.x, (int64_t)min(max(tb + i - (W - 1), r.lo), r.hi - 1) * p.ldx + me.col, xr[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) get<float, V>(p.dy, (int64_t)min(tb + i, r.hi - 1) * p.lddy + me.col, g[i]);
    int pos[N];
    int64_t st[N];
    if constexpr (!INSIDE) {
      places<N, true>(at, tb, tb, r.hi, pos, st);
#pragma unroll
      for (int i = 0; i < N; ++i) first_states<T, W, V>(p, pos[i], st[i], me.col, sv[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float win[W][V];
      window<W, V>(xr, sv[INSIDE ? 0 : i], i, INSIDE ? W : pos[i], win);
      const bool on = i < TR && tb + i < me.t1;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float a = b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) a = fmaf(w[j][v], win[j][v], a);
        const float s = p.act ? dsilu_(a) : 1.f;
        g[i][v] = INSIDE || tb + i < r.hi ? g[i][v] * s : 0.f;
        if (on) {
          db[v] += g[i][v];
#pragma unroll
          for (int j = 0; j < W; ++j) dw[j][v] = fmaf(g[i][v], win[j][v], dw[j][v]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TR; ++i) {
      if (tb + i >= me.t1) break;
      float dx[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        dx[v] = w[W - 1][v] * g[i][v];
#pragma unroll
        for (int k = 1; k < W; ++k) {
          const bool same = INSIDE || (tb + i + k < r.hi && pos[i + k] >= k);
          dx[v] = same ? fmaf(w[W - 1 - k][v], g[i + k][v], dx[v]) : dx[v];
        }
      }
      if (me.mine) put<float, V>(p.dx, (int64_t)(tb + i) * p.lddx + me.col, dx);
    }
  };
  for (int tb = me.t0; tb < me.t1; tb += TR) {
    while (at.beg > tb) at.prev();
    while (tb >= at.end && at.s + 1 < at.n) at.next();
    if (tb - at.beg >= W - 1 && tb + N <= at.end) tile(tb, std::true_type{});
    else tile(tb, std::false_type{});
  }
  if (me.mine) {
    float* part = p.part + (int64_t)me.chunk * (W + 1) * p.d + me.col;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int j = 0; j < W; ++j) part[(int64_t)j * p.d + v] = dw[j][v];
      part[(int64_t)W * p.d + v] = db[v];
    }
  }
}

// Single rows: a thread per row and V channels.
template <typename T, int W, int V>
__global__ __launch_bounds__(256) void k_conv_step(ConvP p, const int32_t* n_rows, int64_t max_rows) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int dv = p.d / V;
  const int64_t row = e / dv;
  if (row >= eff_count(max_rows, n_rows)) return;
  const int ch = (int)(e % dv) * V;
  const int64_t k = seq_slot(p.q.slot, p.q.n_slots, row);
  float v[W][V], w[W][V], a[V];
#pragma unroll
  for (int j = 0; j < W; ++j) {
#pragma unroll
    for (int u = 0; u < V; ++u) v[j][u] = 0.f;
    if (j == W - 1) get<T, V>(p.x, row * p.ldx + ch, v[j]);
    else if (p.st_in && k >= 0) get<T, V>(p.st_in, (k * (W - 1) + j) * p.d + ch, v[j]);
    get<T, V>(p.w, (int64_t)j * p.d + ch, w[j]);
  }
#pragma unroll
  for (int u = 0; u < V; ++u) {
    a[u] = p.b ? p.b[ch + u] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) a[u] = fmaf(w[j][u], v[j][u], a[u]);
    if (p.act) a[u] = silu_(a[u]);
  }
  if (p.st_out && k >= 0) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) put<T, V>(p.st_out, (k * (W - 1) + j) * p.d + ch, v[j + 1]);
  }
  put<T, V>(p.y, row * p.ldy + ch, a);
}

// ------------------------------------------------------------------ host

// Rows of a wave's chunk: enough chunks for about 8,192 waves (two channels a lane: 4,096).  32,768 x 2,048 forward: 102 us
// with half of them, 77 with twice as many; backward 169, 173 and 176, its sums over chunks 5, 9 and 17.
int conv_chunk(int64_t rows, int d) {
  const int64_t waves = std::max<int64_t>(1, 8192 / cdiv(d, 64));
  return (int)(cdiv(cdiv(std::max<int64_t>(rows, 1), waves), TR) * TR);
}

// Whether groups of V channels are aligned.  A lane has two where they are: forward 75 us against 124 with one (77 with
// four), backward 173 against 168 (32,768 rows x 2,048, bfloat16).  Single rows take four channels a thread from 2^20 of
// them on: 4,000 x 2,048 38 us against 46 with two, 52 and more with one.
bool aligned(int V, const mtgnn_conv_dims* d, std::initializer_list<const void*> ps, std::initializer_list<const float*> fs,
             std::initializer_list<int64_t> lds) {
  const uintptr_t a = V * (d->dtype == MTGNN_BF16 ? 2 : 4);
  if (d->d % V) return false;
  for (const void* p : ps)
    if ((uintptr_t)p % a) return false;
  for (const float* p : fs)
    if ((uintptr_t)p % (4 * V)) return false;
  for (int64_t l : lds)
    if (l % V) return false;
  return true;
}

template <typename F>
void conv_variant(const mtgnn_conv_dims* d, int V, F f) {
  const auto by = [&](auto t) {
    using T = decltype(t);
    const auto wide = [&](auto v) {
      constexpr int V = decltype(v)::value;
      if (d->width == 2) f.template operator()<T, 2, V>();
      else if (d->width == 3) f.template operator()<T, 3, V>();
      else f.template operator()<T, 4, V>();
    };
    if (V == 4) wide(std::integral_constant<int, 4>{});
    else if (V == 2) wide(std::integral_constant<int, 2>{});
    else wide(std::integral_constant<int, 1>{});
  };
  if (d->dtype == MTGNN_BF16) by(uint16_t{});
  else by(float{});
}

struct LaunchConv {
  const ConvP& p;
  unsigned grid;
  hipStream_t s;
  template <typename T, int W, int V> void operator()() const {
    if constexpr (V < 4) k_conv<T, W, V><<<grid, 256, 0, s>>>(p);
  }
};
struct LaunchState {
  const ConvP& p;
  unsigned grid;
  hipStream_t s;
  template <typename T, int W, int V> void operator()() const {
    if constexpr (V == 1) k_conv_state<T, W><<<grid, 256, 0, s>>>(p);
  }
};
struct LaunchConvBack {
  const ConvP& p;
  unsigned grid;
  hipStream_t s;
  template <typename T, int W, int V> void operator()() const {
    if constexpr (V < 4) k_conv_back<T, W, V><<<grid, 256, 0, s>>>(p);
  }
};
struct LaunchConvStep {
  const ConvP& p;
  const int32_t* n_rows;
  int64_t max_rows;
  unsigned grid;
  hipStream_t s;
  template <typename T, int W, int V> void operator()() const {
    k_conv_step<T, W, V><<<grid, 256, 0, s>>>(p, n_rows, max_rows);
  }
};

ConvP conv_params(const mtgnn_seqs* q, const void* x, int64_t ldx, const void* w, const float* b,
                  const mtgnn_conv_dims* d) {
  ConvP p{};
  if (q) p.q = seqs_of(q);
  p.x = x; p.w = w; p.b = b; p.ldx = ldx; p.d = d->d; p.act = d->act;
  return p;
}

}  // namespace

size_t conv_save(const mtgnn_conv_dims* d, int64_t max_seq) {
  return (size_t)max_seq * (d->width - 1) * d->d * (d->dtype == MTGNN_BF16 ? 2 : 4);
}
size_t conv_ws(const mtgnn_conv_dims* d, int64_t rows) {
  return (size_t)cdiv(std::max<int64_t>(rows, 1), conv_chunk(rows, d->d)) * (d->width + 1) * d->d * 4;
}

mtgnn_status conv_impl(const mtgnn_seqs* q, const void* x, int64_t ldx, const void* w, const float* b,
                       const mtgnn_conv_dims* d, const void* state_in, void* state_out, void* y, int64_t ldy,
                       void* save, hipStream_t s) {
  ConvP p = conv_params(q, x, ldx, w, b, d);
  p.st_in = state_in; p.st_out = state_out; p.save = save; p.y = y; p.ldy = ldy;
  const int V = aligned(2, d, {x, w, y, state_in}, {}, {ldx, ldy}) ? 2 : 1;
  p.ch = conv_chunk(q->max_rows, d->d);
  p.tiles = (int)cdiv(d->d, 64 * V);
  conv_variant(d, V, LaunchConv{p, (unsigned)(cdiv(cdiv(q->max_rows, p.ch), 4) * p.tiles), s});
  MTGNN_CHECK_LAUNCH("conv");
  if (state_out || save) {
    conv_variant(d, 1, LaunchState{p, (unsigned)cdiv(q->max_seq * d->d, 256), s});
    MTGNN_CHECK_LAUNCH("conv_state");
  }
  return MTGNN_OK;
}

mtgnn_status conv_bwd_impl(const mtgnn_seqs* q, const float* dy, int64_t lddy, const void* x, int64_t ldx,
                           const void* w, const float* b, const mtgnn_conv_dims* d, const void* save, float* dx,
                           int64_t lddx, float* dw, float* db, void* ws, hipStream_t s) {
  ConvP p = conv_params(q, x, ldx, w, b, d);
  p.st_in = save; p.dy = dy; p.lddy = lddy; p.dx = dx; p.lddx = lddx; p.part = (float*)ws;
  const int V = aligned(2, d, {x, w, save}, {dy, dx}, {ldx, lddy, lddx}) ? 2 : 1;
  p.ch = conv_chunk(q->max_rows, d->d);
  p.tiles = (int)cdiv(d->d, 64 * V);
  conv_variant(d, V, LaunchConvBack{p, (unsigned)(cdiv(cdiv(q->max_rows, p.ch), 4) * p.tiles), s});
  MTGNN_CHECK_LAUNCH("conv_back");
  const int64_t wd = (int64_t)d->width * d->d;
  k_sum_parts<<<(unsigned)cdiv(wd + d->d, 16), 256, 0, s>>>(p.q, p.ch, 0, p.part, wd + d->d, wd, dw, d->d, db, nullptr);
  MTGNN_CHECK_LAUNCH("conv_sum_parts");
  return MTGNN_OK;
}

mtgnn_status conv_step_impl(const int32_t* slot, const int32_t* n_rows, int64_t max_rows, int64_t n_slots,
                            const void* x, int64_t ldx, const void* w, const float* b, const mtgnn_conv_dims* d,
                            const void* state_in, void* state_out, void* y, int64_t ldy, hipStream_t s) {
  ConvP p = conv_params(nullptr, x, ldx, w, b, d);
  p.q.slot = slot; p.q.n_slots = n_slots;
  p.st_in = state_in; p.st_out = state_out; p.y = y; p.ldy = ldy;
  const auto by = [&](int V) { return aligned(V, d, {x, w, y, state_in, state_out}, {}, {ldx, ldy}); };
  const int V = max_rows * d->d >= (int64_t(1) << 20) && by(4) ? 4 : by(2) ? 2 : 1;
  conv_variant(d, V, LaunchConvStep{p, n_rows, max_rows, (unsigned)cdiv(max_rows * (d->d / V), 256), s});
  MTGNN_CHECK_LAUNCH("conv_step");
  return MTGNN_OK;
}

}  // namespace mtgnn
