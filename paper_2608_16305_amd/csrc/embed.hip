// Rows of a table by id, scaled, and the table's gradient:
//   y_r = scale table[id_r],   dtable_i = scale sum of dy_r over the rows r with id_r = i.
// An id that is no row of the table gives a row of zeros and takes part in no gradient.
//
// Both are bound by memory.  The gradient is dense: every row of it is written once, as a sum over the rows that carry its id,
// in their order (no float atomics: the result does not depend on scheduling).  The rows are put in the order of their ids first,
// which moves eight bytes of a row of d: one or two passes, each a histogram of tiles and a scatter that keeps the rows' order
// within a digit of up to 13 bits, so two launches a pass where a sort by 8-bit digits takes three, and no rule by which many rows
// of one id would fall to one block.  Ids with many rows are summed in runs that other threads work on at the same time.  (32,768
// rows of 50,000 x 1,024: a pass 11 us, each id's place 8, the sums 78, 339 MB at 4.3 TB/s, the
// runs' join 6.)
#include <algorithm>

#include "ops.h"
#include "words.h"

namespace mtgnn {

namespace {

constexpr int NT = 256;
constexpr int IDS = 4;      // ids that a thread sums

// 16 bytes a thread (four a thread, requested together, took as long).  32,768 rows of 50,000 x 1,024 in bfloat16: 26 us, 134 MB at
// 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(NT) void k_embed(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const T* table,
                                              int64_t n, int d, float scale, T* y, int64_t ldy) {
  constexpr int V = 16 / sizeof(T);
  const uint32_t dv = (uint32_t)cdiv(d, V), e = blockIdx.x * NT + threadIdx.x;
  const int64_t r = e / dv;
  const int c = (int)(e % dv) * V;
  if (r >= eff_count(max_rows, n_rows)) return;
  const int64_t id = ids[r];
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.f;
  if (id >= 0 && id < n) load_some(table + id * d + c, d - c, v);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] *= scale;
  store_some(y + r * ldy + c, d - c, v);
}

// --------------------------------------------------------------------------- rows in the order of their ids

// 64 tiles at most: a block of the scatter adds up a digit's counts of all of them.  32, 64, 128 and 256 at most, the forward with the
// gradient, us: 200,000 rows of 9,000 x 200 in float32 169, 151, 145 and 149; 200,000 of 1,000,000 x 60 219, 202, 196 and 201; 150,000
// of 60,000 x 100 100, 89, 87 and 87; 70,000 of 8,192 x 100 84, 78, 90 and 88; up to 65,536 rows they are the same.
constexpr int ST = 1024, MAX_DIGITS = 8192, MAX_TILES = 64;
constexpr int MANY = 64;     // ids of a block whose runs all of its threads list

// What the gradient's kernels share, in the workspace.
struct Groups {
  int64_t rows, n, per;      // rows, ids, rows of a tile (a block of the passes)
  int tiles, low;            // low: bits of an id that the first of two passes sorts by (0: one pass)
  int light;                 // rows that one thread sums (per column): of an id, of a run of one with more
  int32_t* hist;             // [tiles][digits]
  int32_t *first, *firsts;   // [digits + 1] first position of each digit of the last pass; the same of the first one
  uint32_t *id[2], *row[2];  // id and row of each position after a pass
  int32_t* off;              // [n + 1] first position of each id
  int32_t* counts;           // [2] runs, heavy ids
  int32_t* run;              // [runs] two each: first and last position
  int32_t* heavy;            // [heavy ids] three each: id, first run, runs
  float* part;               // [runs][d]
};
// A pass: position i of its input has an id, or (the first pass) is a row that may have none.
struct Pass {
  const uint32_t *id, *row;  // NULL: the first pass, `ids`
  const int32_t *ids, *n_rows, *count;   // count: positions of the input of the second
  int shift, digits;
  uint32_t mask;
  uint32_t *to_id, *to_row;
  int32_t* first;
};
__device__ __forceinline__ int64_t length(const Groups& g, const Pass& p) {
  return p.count ? (int64_t)*p.count : eff_count(g.rows, p.n_rows);
}
__device__ __forceinline__ bool get(const Groups& g, const Pass& p, int64_t i, int64_t end, uint32_t& id) {
  id = i < end ? (p.id ? p.id[i] : (uint32_t)p.ids[i]) : 0xffffffffu;
  return id < (uint64_t)g.n;
}

// The lanes of a wave that have the same key (of `bits` bits), of those that have one.
__device__ __forceinline__ uint64_t same_key(bool have, uint32_t key, int bits) {
  uint64_t peers = __ballot(have);
  for (int b = 0; b < bits; ++b) {
    const bool bit = key >> b & 1;
    const uint64_t m = __ballot(bit);
    peers &= bit ? m : ~m;
  }
  return have ? peers : 0;
}
__device__ __forceinline__ int lower_lanes(uint64_t m) { return __popcll(m & ((uint64_t(1) << (threadIdx.x & 63)) - 1)); }

// Exclusive sums over a block's threads; total: of all.
template <int THREADS>
__device__ __forceinline__ int block_exclusive(int v, int& total, int* s) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(inc, o, 64);
    if (lane >= o) inc += t;
  }
  if (lane == 63) s[wid] = inc;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    before += w < wid ? s[w] : 0;
    total += s[w];
  }
  __syncthreads();
  return before + inc - v;
}

__global__ __launch_bounds__(ST) void k_embed_hist(Groups g, Pass p) {
  __shared__ int h[MAX_DIGITS];
  const int64_t i0 = blockIdx.x * g.per, end = min(length(g, p), i0 + g.per);
  if (blockIdx.x == 0 && threadIdx.x < 2) g.counts[threadIdx.x] = 0;
  for (int b = threadIdx.x; b < p.digits; b += ST) h[b] = 0;
  __syncthreads();
  for (int64_t i = i0 + threadIdx.x; i < end; i += ST) {
    uint32_t id;
    if (get(g, p, i, end, id)) atomicAdd(&h[id >> p.shift & p.mask], 1);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < p.digits; b += ST) g.hist[(int64_t)blockIdx.x * p.digits + b] = h[b];
}

// A tile's rows to their digits, behind those of the tiles before it; waves of a tile in turn, so that the order stays.
__global__ __launch_bounds__(ST) void k_embed_scatter(Groups g, Pass p) {
  __shared__ int at[MAX_DIGITS];
  __shared__ int s[ST / 64];
  const int64_t i0 = blockIdx.x * g.per, end = min(length(g, p), i0 + g.per);
  const int wid = threadIdx.x >> 6;
  uint32_t id;
  bool have = get(g, p, i0 + threadIdx.x, end, id);
  int base = 0;
  for (int b0 = 0; b0 < p.digits; b0 += ST) {
    const int b = b0 + threadIdx.x;
    int before = 0, all = 0, total;
    if (b < p.digits)
#pragma unroll 8
      for (int t = 0; t < g.tiles; ++t) {
        const int v = g.hist[(int64_t)t * p.digits + b];
        before += t < (int)blockIdx.x ? v : 0;
        all += v;
      }
    const int from = base + block_exclusive<ST>(all, total, s);
    if (b < p.digits) {
      at[b] = from + before;
      if (blockIdx.x == 0) p.first[b] = from;
    }
    base += total;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.first[p.digits] = base;
  __syncthreads();
  const int bits = 32 - __clz(max(1, p.digits - 1));
  for (int64_t c = i0; c < end; c += ST) {
    const int64_t i = c + threadIdx.x;
    const uint32_t b = have ? id >> p.shift & p.mask : 0u;
    const uint32_t r = have ? (p.row ? p.row[i] : (uint32_t)i) : 0u;
    const uint64_t peers = same_key(have, b, bits);
    const int rank = lower_lanes(peers);
    int pos = 0;
    for (int w = 0; w < ST / 64; ++w) {
      if (w == wid && have) {
        pos = at[b] + rank;
        if (rank + 1 == __popcll(peers)) at[b] = pos + 1;   // the last of them
      }
      __syncthreads();
    }
    if (have) {
      p.to_id[pos] = id;
      p.to_row[pos] = r;
    }
    have = get(g, p, i + ST, end, id);
  }
}

// Every id's first position (a search among those that share its high digit), and the runs of those with more than `light` rows.
__global__ __launch_bounds__(NT) void k_embed_bounds(Groups g, const uint32_t* key) {
  __shared__ int s[NT / 64], base[2], many[MANY][3], n_many;
  const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x;
  const auto first_of = [&](int64_t id) {
    int lo = g.first[id >> g.low], hi = id < g.n ? g.first[(id >> g.low) + 1] : lo;
    while (lo < hi) {
      const int m = (lo + hi) >> 1;
      if (key[m] < id) lo = m + 1;
      else hi = m;
    }
    return lo;
  };
  int from = 0, count = 0;
  if (i <= g.n) g.off[i] = from = i < g.n ? first_of(i) : g.first[(g.n - 1 >> g.low) + 1];
  if (i < g.n) count = (i + 1 < g.n ? first_of(i + 1) : g.first[(g.n - 1 >> g.low) + 1]) - from;
  const int light = g.light, runs = count > light ? (count + light - 1) / light : 0;
  int all, all_runs;
  const int h = block_exclusive<NT>(runs > 0, all, s), f = block_exclusive<NT>(runs, all_runs, s);
  if (all == 0) return;
  if (threadIdx.x == 0) {   // (places, not order)
    n_many = 0;
    base[0] = atomicAdd(g.counts, all_runs);
    base[1] = atomicAdd(g.counts + 1, all);
  }
  __syncthreads();
  if (runs) {
    const int o = base[1] + h;
    g.heavy[3 * o] = (int32_t)i;
    g.heavy[3 * o + 1] = base[0] + f;
    g.heavy[3 * o + 2] = runs;
    // those of many runs by the whole block, below
    const int q = runs > 4 ? atomicAdd(&n_many, 1) : MANY;
    if (q < MANY) {
      many[q][0] = base[0] + f;
      many[q][1] = from;
      many[q][2] = count;
    } else {
      for (int k = 0; k < runs; ++k) {
        g.run[2 * (base[0] + f + k)] = from + k * light;
        g.run[2 * (base[0] + f + k) + 1] = from + min(count, (k + 1) * light);
      }
    }
  }
  __syncthreads();
  for (int q = 0; q < min(n_many, MANY); ++q)
    for (int k = threadIdx.x; k * light < many[q][2]; k += NT) {
      g.run[2 * (many[q][0] + k)] = many[q][1] + k * light;
      g.run[2 * (many[q][0] + k) + 1] = many[q][1] + min(many[q][2], (k + 1) * light);
    }
}

// --------------------------------------------------------------------------- sums

// s += the rows at positions a .. b - 1, in their order.
__device__ __forceinline__ void add_rows(float (&s)[4], const uint32_t* row, int a, int b, const float* dy, int64_t ld, int n) {
  for (int k = a; k < b; k += 8) {
    float v[8][4];
    uint32_t r[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) r[u] = row[min(k + u, b - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) load_some(dy + (int64_t)r[u] * ld, n, v[u]);
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = k + u < b ? s[j] + v[u][j] : s[j];
  }
}

// Four columns of IDS neighbouring ids (those with at most `light` rows), or of a run: blocks from id_blocks on.  An id's first two
// rows are requested for all of them together.
__global__ __launch_bounds__(NT) void k_embed_sum(Groups g, const uint32_t* row, const float* dy, int64_t lddy, int d, float scale,
                                                  int64_t id_blocks, float* dtable) {
  const int dv = (int)cdiv(d, 4);
  const bool runs = blockIdx.x >= id_blocks;
  const uint32_t e = (uint32_t)(blockIdx.x - (runs ? id_blocks : 0)) * NT + threadIdx.x;
  const int64_t i = e / dv;
  const int c = (int)(e % dv) * 4, n = d - c;
  dy += c;
  if (runs) {
    if (i >= g.counts[0]) return;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    add_rows(s, row, g.run[2 * i], g.run[2 * i + 1], dy, lddy, n);
    store_some(g.part + i * d + c, n, s);
    return;
  }
  const int64_t id = i * IDS;
  if (id >= g.n) return;
  int off[IDS + 1];
#pragma unroll
  for (int u = 0; u <= IDS; ++u) off[u] = g.off[min(id + u, g.n)];
  uint32_t r[IDS][2];
  float v[IDS][2][4];
#pragma unroll
  for (int u = 0; u < IDS; ++u)
#pragma unroll
    for (int k = 0; k < 2; ++k) r[u][k] = off[u] + k < off[u + 1] ? row[off[u] + k] : 0u;
#pragma unroll
  for (int u = 0; u < IDS; ++u)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[u][k][j] = 0.f;
      if (off[u] + k < off[u + 1]) load_some(dy + (int64_t)r[u][k] * lddy, n, v[u][k]);
    }
#pragma unroll
  for (int u = 0; u < IDS; ++u) {
    const int count = off[u + 1] - off[u];
    if (id + u >= g.n || count > g.light) continue;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = k < count ? s[j] + v[u][k][j] : s[j];
    if (count > 2) add_rows(s, row, off[u] + 2, off[u + 1], dy, lddy, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] *= scale;
    store_some(dtable + (id + u) * d + c, n, s);
  }
}

// The runs of a heavy id: a block has 16 times four columns of one, and 16 threads to each, which take every 16th run.
__global__ __launch_bounds__(NT) void k_embed_join(Groups g, int d, float scale, float* dtable) {
  __shared__ float s[16][16][4];
  const int cb = (int)cdiv(d, 64), h = blockIdx.x / cb, j16 = threadIdx.x & 15, k16 = threadIdx.x >> 4;
  const int c = (int)(blockIdx.x % cb) * 64 + j16 * 4, n = d - c;
  if (h >= g.counts[1]) return;
  const int first = g.heavy[3 * h + 1], runs = g.heavy[3 * h + 2];
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (n > 0)
#pragma unroll 4
    for (int k = k16; k < runs; k += 16) {
      float w[4];
      load_some(g.part + (int64_t)(first + k) * d + c, n, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += w[j];
    }
#pragma unroll
  for (int j = 0; j < 4; ++j) s[k16][j16][j] = v[j];
  __syncthreads();
  if (k16 || n <= 0) return;
#pragma unroll
  for (int k = 1; k < 16; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += s[k][j16][j];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] *= scale;
  store_some(dtable + (int64_t)g.heavy[3 * h] * d + c, n, v);
}

size_t al(size_t b) { return (b + 255) & ~size_t(255); }
// Shorter runs where there is little work for threads to share: 16 and 32, us, with the forward, 8,000 rows of 100,000 x 100 in
// float32 43.9 and 46.6, 32,768 of 50,000 x 1,024 in bfloat16 143 and 138, 200,000 of 9,000 x 200 126 and 112 (64: 143 and 111).
int light_rows(int64_t rows, int d) { return rows * cdiv(d, 4) >= int64_t(1) << 20 ? 32 : 16; }
int64_t most_heavy(int64_t rows, int d) { return rows / (light_rows(rows, d) + 1); }
int64_t most_runs(int64_t rows, int d) { return rows / light_rows(rows, d) + most_heavy(rows, d); }

// One pass where every id can be a digit, else two of about half of an id's bits.
void lay_out(Groups& g, int64_t rows, int64_t n) {
  g.rows = rows;
  g.n = n;
  g.per = std::max<int64_t>(ST, cdiv(cdiv(rows, MAX_TILES), ST) * ST);
  g.tiles = (int)cdiv(rows, g.per);
  g.low = n <= MAX_DIGITS ? 0 : bits_for(n - 1) / 2;
}
size_t place(Groups& g, int d, char* w) {
  char* const start = w;
  const auto take = [&](size_t bytes) {
    char* p = w;
    w += al(bytes);
    return p;
  };
  const size_t high = (size_t)cdiv(g.n, int64_t(1) << g.low), low = g.low ? size_t(1) << g.low : 0;
  g.hist = (int32_t*)take(4 * (size_t)g.tiles * std::max(high, low));
  g.first = (int32_t*)take(4 * (high + 1));
  g.firsts = (int32_t*)take(4 * (low + 1));
  for (int k = 0; k < 2; ++k) {
    g.id[k] = (uint32_t*)take(4 * g.rows);
    g.row[k] = (uint32_t*)take(4 * g.rows);
  }
  g.off = (int32_t*)take(4 * (g.n + 1));
  g.counts = (int32_t*)take(8);
  g.light = light_rows(g.rows, d);
  g.run = (int32_t*)take(8 * most_runs(g.rows, d));
  g.heavy = (int32_t*)take(12 * most_heavy(g.rows, d));
  g.part = (float*)take(4 * most_runs(g.rows, d) * d);
  return (size_t)(w - start);
}

}  // namespace

bool embed_fits(const mtgnn_embedding_dims* d, int64_t rows, bool back) {
  constexpr int64_t MAX = (int64_t(1) << 32) - 2 * NT;
  if (!back) return rows * cdiv(d->d, d->dtype == MTGNN_BF16 ? 8 : 4) <= MAX;
  const int64_t dv = cdiv(d->d, 4);
  return d->n <= (int64_t)MAX_DIGITS * MAX_DIGITS && cdiv(cdiv(d->n, IDS) * dv, NT) * NT + most_runs(rows, d->d) * dv <= MAX &&
         most_heavy(rows, d->d) * cdiv(d->d, 64) * NT <= MAX;
}

size_t embed_ws(const mtgnn_embedding_dims* d, int64_t rows) {
  Groups g;
  lay_out(g, rows, d->n);
  return place(g, d->d, nullptr);
}

template <typename T>
mtgnn_status embed_t(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const T* table, const mtgnn_embedding_dims* d,
                     T* y, int64_t ldy, hipStream_t s) {
  const int64_t items = max_rows * cdiv(d->d, 16 / (int)sizeof(T));
  k_embed<T><<<(unsigned)cdiv(items, NT), NT, 0, s>>>(ids, n_rows, max_rows, table, d->n, d->d, d->scale, y, ldy);
  MTGNN_CHECK_LAUNCH("embed");
  return MTGNN_OK;
}

mtgnn_status embed_impl(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const void* table,
                        const mtgnn_embedding_dims* d, void* y, int64_t ldy, hipStream_t s) {
  if (d->dtype == MTGNN_BF16) return embed_t(ids, n_rows, max_rows, (const uint16_t*)table, d, (uint16_t*)y, ldy, s);
  return embed_t(ids, n_rows, max_rows, (const float*)table, d, (float*)y, ldy, s);
}

mtgnn_status embed_bwd_impl(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const float* dy, int64_t lddy,
                            const mtgnn_embedding_dims* d, float* dtable, void* ws, hipStream_t s) {
  Groups g;
  lay_out(g, max_rows, d->n);
  place(g, d->d, (char*)ws);
  const auto pass = [&](const Pass& p) -> mtgnn_status {
    k_embed_hist<<<(unsigned)g.tiles, ST, 0, s>>>(g, p);
    MTGNN_CHECK_LAUNCH("embed_hist");
    k_embed_scatter<<<(unsigned)g.tiles, ST, 0, s>>>(g, p);
    MTGNN_CHECK_LAUNCH("embed_scatter");
    return MTGNN_OK;
  };
  const int high = (int)cdiv(d->n, int64_t(1) << g.low), last = g.low ? 1 : 0;
  if (g.low) {
    const int digits = 1 << g.low;
    MTGNN_TRY(pass(Pass{nullptr, nullptr, ids, n_rows, nullptr, 0, digits, (uint32_t)digits - 1, g.id[0], g.row[0], g.firsts}));
    MTGNN_TRY(pass(Pass{g.id[0], g.row[0], nullptr, nullptr, g.firsts + digits, g.low, high, ~0u, g.id[1], g.row[1], g.first}));
  } else {
    MTGNN_TRY(pass(Pass{nullptr, nullptr, ids, n_rows, nullptr, 0, high, ~0u, g.id[0], g.row[0], g.first}));
  }
  k_embed_bounds<<<(unsigned)cdiv(d->n + 1, NT), NT, 0, s>>>(g, g.id[last]);
  MTGNN_CHECK_LAUNCH("embed_bounds");
  const int64_t dv = cdiv(d->d, 4), id_blocks = cdiv(cdiv(d->n, IDS) * dv, NT);
  const int64_t run_blocks = cdiv(most_runs(max_rows, d->d) * dv, NT);
  k_embed_sum<<<(unsigned)(id_blocks + run_blocks), NT, 0, s>>>(g, g.row[last], dy, lddy, d->d, d->scale, id_blocks,
                                                                dtable);
  MTGNN_CHECK_LAUNCH("embed_sum");
  if (most_heavy(max_rows, d->d) > 0) {
    k_embed_join<<<(unsigned)(most_heavy(max_rows, d->d) * cdiv(d->d, 64)), NT, 0, s>>>(g, d->d, d->scale, dtable);
    MTGNN_CHECK_LAUNCH("embed_join");
  }
  return MTGNN_OK;
}

}  // namespace mtgnn
