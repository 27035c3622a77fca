// Rows of a table by id, scaled, and the table's gradient:
//   y_r = scale table[id_r],   dtable_i = scale sum of dy_r over the rows r with id_r = i.
// An id that is no row of the table gives a row of zeros and takes part in no gradient.
//
// Both are bound by memory.  The gradient is dense: every row of it is written once, as a sum over the rows that carry its id,
// in their order (no float atomics: the result does not depend on scheduling).  The rows are grouped by id first, which moves
// four bytes of a row of d; ids with more than LIGHT rows are summed in runs that other threads work on at the same time.
#include <algorithm>

#include "ops.h"
#include "words.h"

namespace mtgnn {

namespace {

constexpr int NT = 256;
constexpr int LIGHT = 32;   // rows of an id that one thread sums (per column)

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

// What the gradient's kernels share, in the workspace.
struct Groups {
  uint32_t *key, *row;       // of each position in the order of ids: the id (n: none), the row
  int32_t* off;              // [n + 1] first position of each id
  int32_t* counts;           // [2] runs, heavy ids
  int32_t* run;              // [runs] two each: first and last position
  int32_t* heavy;            // [heavy ids] three each: id, first run, runs
  float* part;               // [runs][d]
};

__global__ __launch_bounds__(NT) void k_embed_keys(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, int64_t n,
                                                   uint32_t* key, uint32_t* row, int32_t* counts) {
  const int64_t r = (int64_t)blockIdx.x * NT + threadIdx.x;
  if (r < 2) counts[r] = 0;
  if (r >= max_rows) return;
  const int64_t id = ids[r];
  key[r] = r < eff_count(max_rows, n_rows) && id >= 0 && id < n ? (uint32_t)id : (uint32_t)n;
  row[r] = (uint32_t)r;
}

__device__ __forceinline__ int64_t lower_bound(const uint32_t* key, int64_t rows, uint32_t id) {
  int64_t lo = 0, hi = rows;
  while (lo < hi) {
    const int64_t m = (lo + hi) >> 1;
    if (key[m] < id) lo = m + 1;
    else hi = m;
  }
  return lo;
}

// Positions in a run of a heavy id of `count` rows: about the root, so that neither the runs nor their sums are long chains.
__device__ __forceinline__ int run_length(int count) {
  return max(LIGHT, ((int)sqrtf((float)count) + LIGHT - 1) / LIGHT * LIGHT);
}

__global__ __launch_bounds__(NT) void k_embed_bounds(Groups g, int64_t rows, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x;
  if (i > n) return;
  const int64_t a = lower_bound(g.key, rows, (uint32_t)i);
  g.off[i] = (int32_t)a;
  if (i == n) return;
  const int count = (int)(lower_bound(g.key, rows, (uint32_t)i + 1) - a);
  if (count <= LIGHT) return;
  const int L = run_length(count), runs = (int)cdiv(count, L);
  const int first = atomicAdd(g.counts, runs), h = atomicAdd(g.counts + 1, 1);   // (places, not order)
  g.heavy[3 * h] = (int32_t)i;
  g.heavy[3 * h + 1] = first;
  g.heavy[3 * h + 2] = runs;
  for (int k = 0; k < runs; ++k) {
    g.run[2 * (first + k)] = (int32_t)a + k * L;
    g.run[2 * (first + k) + 1] = (int32_t)a + min(count, (k + 1) * L);
  }
}

// Threads below n ids x columns: the ids with at most LIGHT rows.  The others: the runs of the heavy ones.
__global__ __launch_bounds__(NT) void k_embed_sum(Groups g, const float* dy, int64_t lddy, int64_t n, int d, float scale,
                                                  int64_t id_blocks, float* dtable) {
  const int dv = (int)cdiv(d, 4);
  const bool runs = blockIdx.x >= id_blocks;
  const uint32_t e = (uint32_t)(blockIdx.x - (runs ? id_blocks : 0)) * NT + threadIdx.x;
  const int64_t i = e / dv;
  const int c = (int)(e % dv) * 4;
  int a, b;
  float* out;
  if (runs) {
    if (i >= g.counts[0]) return;
    a = g.run[2 * i];
    b = g.run[2 * i + 1];
    out = g.part + i * d + c;
    scale = 1.f;
  } else {
    if (i >= n) return;
    a = g.off[i];
    b = g.off[i + 1];
    if (b - a > LIGHT) return;
    out = dtable + i * d + c;
  }
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = a; k < b; k += 4) {
    float v[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) load_some(dy + (int64_t)g.row[min(k + u, b - 1)] * lddy + c, d - c, v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = k + u < b ? s[j] + v[u][j] : s[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) s[j] *= scale;
  store_some(out, d - c, s);
}

__global__ __launch_bounds__(NT) void k_embed_heavy(Groups g, int d, float scale, float* dtable) {
  const uint32_t dv = (uint32_t)cdiv(d, 4), e = blockIdx.x * NT + threadIdx.x;
  const int64_t h = e / dv;
  const int c = (int)(e % dv) * 4;
  if (h >= g.counts[1]) return;
  const int64_t id = g.heavy[3 * h];
  const int first = g.heavy[3 * h + 1], runs = g.heavy[3 * h + 2];
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < runs; k += 4) {
    float v[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) load_some(g.part + (int64_t)(first + min(k + u, runs - 1)) * d + c, d - c, v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = k + u < runs ? s[j] + v[u][j] : s[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) s[j] *= scale;
  store_some(dtable + id * d + c, d - c, s);
}

size_t al(size_t b) { return (b + 255) & ~size_t(255); }
int64_t most_heavy(int64_t rows) { return rows / (LIGHT + 1); }
int64_t most_runs(int64_t rows) { return rows / LIGHT + most_heavy(rows); }

}  // namespace

bool embed_fits(const mtgnn_embedding_dims* d, int64_t rows, bool back) {
  constexpr int64_t MAX = (int64_t(1) << 32) - 2 * NT;
  const int64_t V = d->dtype == MTGNN_BF16 ? 8 : 4;
  if (!back) return rows * cdiv(d->d, V) <= MAX;
  return cdiv(d->n * cdiv(d->d, 4), NT) * NT + most_runs(rows) * cdiv(d->d, 4) <= MAX;
}

size_t embed_ws(const mtgnn_embedding_dims* d, int64_t rows) {
  return 2 * al(4 * rows) + al(4 * (d->n + 1)) + 256 + al(8 * most_runs(rows)) + al(12 * most_heavy(rows)) +
         al(4 * most_runs(rows) * d->d) + radix_sort_ws_bytes(rows);
}

mtgnn_status embed_impl(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const void* table,
                        const mtgnn_embedding_dims* d, void* y, int64_t ldy, hipStream_t s) {
  const bool bf = d->dtype == MTGNN_BF16;
  const unsigned grid = (unsigned)cdiv(max_rows * cdiv(d->d, bf ? 8 : 4), NT);
  if (bf) k_embed<<<grid, NT, 0, s>>>(ids, n_rows, max_rows, (const uint16_t*)table, d->n, d->d, d->scale, (uint16_t*)y, ldy);
  else k_embed<<<grid, NT, 0, s>>>(ids, n_rows, max_rows, (const float*)table, d->n, d->d, d->scale, (float*)y, ldy);
  MTGNN_CHECK_LAUNCH("embed");
  return MTGNN_OK;
}

mtgnn_status embed_bwd_impl(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const float* dy, int64_t lddy,
                            const mtgnn_embedding_dims* d, float* dtable, void* ws, size_t ws_bytes, hipStream_t s) {
  char* w = (char*)ws;
  const auto take = [&](size_t bytes) {
    char* p = w;
    w += al(bytes);
    return p;
  };
  Groups g;
  g.key = (uint32_t*)take(4 * max_rows);
  g.row = (uint32_t*)take(4 * max_rows);
  g.off = (int32_t*)take(4 * (d->n + 1));
  g.counts = (int32_t*)take(8);
  g.run = (int32_t*)take(8 * most_runs(max_rows));
  g.heavy = (int32_t*)take(12 * most_heavy(max_rows));
  g.part = (float*)take(4 * most_runs(max_rows) * d->d);
  k_embed_keys<<<(unsigned)cdiv(max_rows, NT), NT, 0, s>>>(ids, n_rows, max_rows, d->n, g.key, g.row, g.counts);
  MTGNN_CHECK_LAUNCH("embed_keys");
  MTGNN_TRY(radix_sort_pairs(&g.key, &g.row, max_rows, bits_for(d->n), w, ws_bytes - (size_t)(w - (char*)ws), s));
  k_embed_bounds<<<(unsigned)cdiv(d->n + 1, NT), NT, 0, s>>>(g, max_rows, d->n);
  MTGNN_CHECK_LAUNCH("embed_bounds");
  const int64_t dv = cdiv(d->d, 4), id_blocks = cdiv(d->n * dv, NT);
  k_embed_sum<<<(unsigned)(id_blocks + cdiv(most_runs(max_rows) * dv, NT)), NT, 0, s>>>(g, dy, lddy, d->n, d->d, d->scale,
                                                                                         id_blocks, dtable);
  MTGNN_CHECK_LAUNCH("embed_sum");
  if (most_heavy(max_rows) > 0) {
    k_embed_heavy<<<(unsigned)cdiv(most_heavy(max_rows) * dv, NT), NT, 0, s>>>(g, d->d, d->scale, dtable);
    MTGNN_CHECK_LAUNCH("embed_heavy");
  }
  return MTGNN_OK;
}

}  // namespace mtgnn
