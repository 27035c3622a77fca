// Layer norm of rows and its backward:
//   m = mean x,  q = (mean (x - m)^2 + eps)^-1/2,  h = (x - m) q,  y = gamma h + beta;
//   g = dy gamma,  dx = q (g - mean g - h mean(g h)) [+ past],  dgamma = sum over rows of dy h,  dbeta = sum of dy.
//
// Bound by memory: a row is read once and kept in registers, so that the squares are of what is left after the mean (a
// single pass of sums of x and x^2 loses the variance of a row that is far from zero).  G lanes work on a row (a wave, or a
// block for wide rows), N times V elements each.  The backward's sums over rows stay in registers while a block walks over
// its rows, and leave once per block.
#include <algorithm>

#include "ops.h"
#include "words.h"

namespace mtgnn {

namespace {

// Sum over the G threads of a row; s: one slot a wave, unused in waves.
template <int G>
__device__ __forceinline__ float row_sum(float v, float* s) {
  v = wave_sum(v);
  if constexpr (G > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) v += s[w];
  }
  return v;
}

template <typename T, int G, int N>
__global__ __launch_bounds__(G == 64 ? 256 : G) void k_norm(const T* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows,
                                                            const float* gamma, const float* beta, int d, float eps, T* y,
                                                            int64_t ldy, float2* stats) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float s[G / 64];
  const int64_t r = G == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int t = threadIdx.x % G;
  if (r >= eff_count(max_rows, n_rows)) return;
  float v[N][V], sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * G + t) * V;
    if (c < d) load_some(x + r * ldx + c, d - c, v[i]);
    else
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) sum += v[i][j];
  const float mean = row_sum<G>(sum, s) / d;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      v[i][j] -= mean;
      sum += (i * G + t) * V + j < d ? v[i][j] * v[i][j] : 0.f;
    }
  const float q = 1.f / sqrtf(row_sum<G>(sum, s) / d + eps);
  if (stats && t == 0) stats[r] = make_float2(mean, q);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * G + t) * V;
    if (c >= d) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) v[i][j] *= q;
    float w[V];
    if (gamma) {
      load_some(gamma + c, d - c, w);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] *= w[j];
    }
    if (beta) {
      load_some(beta + c, d - c, w);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] += w[j];
    }
    store_some(y + r * ldy + c, d - c, v[i]);
  }
}

// Rows wider than a block's registers: read again for each pass (from the L2 where they fit it).
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_wide(const T* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows,
                                                    const float* gamma, const float* beta, int d, float eps, T* y,
                                                    int64_t ldy, float2* stats) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float s[16];
  const int64_t r = blockIdx.x;
  if (r >= eff_count(max_rows, n_rows)) return;
  x += r * ldx;
  float sum = 0.f, v[V];
  for (int c = threadIdx.x * V; c < d; c += 1024 * V) {
    load_some(x + c, d - c, v);
#pragma unroll
    for (int j = 0; j < V; ++j) sum += v[j];
  }
  const float mean = row_sum<1024>(sum, s) / d;
  sum = 0.f;
  for (int c = threadIdx.x * V; c < d; c += 1024 * V) {
    load_some(x + c, d - c, v);
#pragma unroll
    for (int j = 0; j < V; ++j) sum += c + j < d ? (v[j] - mean) * (v[j] - mean) : 0.f;
  }
  const float q = 1.f / sqrtf(row_sum<1024>(sum, s) / d + eps);
  if (stats && threadIdx.x == 0) stats[r] = make_float2(mean, q);
  for (int c = threadIdx.x * V; c < d; c += 1024 * V) {
    load_some(x + c, d - c, v);
    float w[V], b[V];
    if (gamma) load_some(gamma + c, d - c, w);
    if (beta) load_some(beta + c, d - c, b);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      v[j] = (v[j] - mean) * q;
      if (gamma) v[j] *= w[j];
      if (beta) v[j] += b[j];
    }
    store_some(y + r * ldy + c, d - c, v);
  }
}

// A team of G threads takes every `teams`-th row.  part: [blocks][2 d], a block's shares of dgamma before those of dbeta.
template <typename T, int G, int N>
__global__ __launch_bounds__(G == 64 ? 256 : G) void k_norm_back(const float* dy, int64_t lddy, const T* x, int64_t ldx,
                                                                 const float2* stats, const int32_t* n_rows,
                                                                 int64_t max_rows, const float* gamma, const float* past,
                                                                 int64_t ldp, int d, float* dx, int64_t lddx, int teams,
                                                                 float* part) {
  constexpr int V = 4;
  __shared__ float2 s[2][G / 64];
  const int64_t rows = eff_count(max_rows, n_rows);
  const int t = threadIdx.x % G;
  const int64_t team = G == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  float dg[N][V], db[N][V], w[N][V];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * G + t) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) dg[i][j] = db[i][j] = 0.f, w[i][j] = 1.f;
    if (gamma && c < d) load_some(gamma + c, d - c, w[i]);
  }
  int turn = 0;
  for (int64_t r = team < teams ? team : rows; r < rows; r += teams, turn ^= 1) {
    const float2 st = stats[r];
    float h[N][V], g[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + t) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) h[i][j] = g[i][j] = 0.f;
      if (c < d) {
        load_some(x + r * ldx + c, d - c, h[i]);
        load_some(dy + r * lddy + c, d - c, g[i]);
      }
    }
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[i][j] = (h[i][j] - st.x) * st.y;
        if ((i * G + t) * V + j >= d) h[i][j] = 0.f;
        dg[i][j] += g[i][j] * h[i][j];
        db[i][j] += g[i][j];
        g[i][j] *= w[i][j];
        a += g[i][j];
        b += g[i][j] * h[i][j];
      }
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (G > 64) {   // (two sets of slots: a wave may be a row ahead)
      if ((threadIdx.x & 63) == 0) s[turn][threadIdx.x >> 6] = make_float2(a, b);
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int k = 0; k < G / 64; ++k) {
        a += s[turn][k].x;
        b += s[turn][k].y;
      }
    }
    a /= d;
    b /= d;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + t) * V;
      if (c >= d) continue;
      float p[V] = {0.f, 0.f, 0.f, 0.f};
      if (past) load_some(past + r * ldp + c, d - c, p);
#pragma unroll
      for (int j = 0; j < V; ++j) p[j] += st.y * (g[i][j] - a - h[i][j] * b);
      store_some(dx + r * lddx + c, d - c, p);
    }
  }
  if (!part) return;
  if constexpr (G == 64) {   // the block's four teams
    __shared__ float4 q[3][2 * N][64];
    const int wid = threadIdx.x >> 6;
    if (wid) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        q[wid - 1][i][t] = make_float4(dg[i][0], dg[i][1], dg[i][2], dg[i][3]);
        q[wid - 1][N + i][t] = make_float4(db[i][0], db[i][1], db[i][2], db[i][3]);
      }
    }
    __syncthreads();
    if (wid) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float4 a = q[w][i][t], b = q[w][N + i][t];
        dg[i][0] += a.x; dg[i][1] += a.y; dg[i][2] += a.z; dg[i][3] += a.w;
        db[i][0] += b.x; db[i][1] += b.y; db[i][2] += b.z; db[i][3] += b.w;
      }
  }
  part += (int64_t)blockIdx.x * 2 * d;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (i * G + t) * V;
    if (c >= d) continue;
    store_some(part + c, d - c, dg[i]);
    store_some(part + d + c, d - c, db[i]);
  }
}

// The blocks' shares: 64 columns a block, four to each of 16 threads, and 32 times 16 threads that take every 32nd share.
__global__ __launch_bounds__(512) void k_norm_join(const float* part, int shares, int d, float* dgamma, float* dbeta) {
  __shared__ float s[32][16][4];
  const int j16 = threadIdx.x & 15, k32 = threadIdx.x >> 4, c = blockIdx.x * 64 + j16 * 4, n = 2 * d - c;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (n > 0)
    for (int k = k32; k < shares; k += 256) {
      float w[8][4];
#pragma unroll
      for (int u = 0; u < 8; ++u) load_some(part + (int64_t)min(k + 32 * u, shares - 1) * 2 * d + c, n, w[u]);
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = k + 32 * u < shares ? v[j] + w[u][j] : v[j];
    }
#pragma unroll
  for (int j = 0; j < 4; ++j) s[k32][j16][j] = v[j];
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int col = blockIdx.x * 64 + threadIdx.x;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) sum += s[k][threadIdx.x >> 2][threadIdx.x & 3];
  if (col < d) {
    if (dgamma) dgamma[col] = sum;
  } else if (col < 2 * d) {
    if (dbeta) dbeta[col - d] = sum;
  }
}

// Rows wider than a block's registers: the row's two sums, then dx; the sums over rows by column afterwards.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_back_wide(const float* dy, int64_t lddy, const T* x, int64_t ldx,
                                                         const float2* stats, const int32_t* n_rows, int64_t max_rows,
                                                         const float* gamma, const float* past, int64_t ldp, int d, float* dx,
                                                         int64_t lddx) {
  __shared__ float s[16];
  const int64_t r = blockIdx.x;
  if (r >= eff_count(max_rows, n_rows)) return;
  const float2 st = stats[r];
  float a = 0.f, b = 0.f, h[4], g[4], w[4] = {1.f, 1.f, 1.f, 1.f};
  const auto get = [&](int c) {
    load_some(x + r * ldx + c, d - c, h);
    load_some(dy + r * lddy + c, d - c, g);
    if (gamma) load_some(gamma + c, d - c, w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      h[j] = c + j < d ? (h[j] - st.x) * st.y : 0.f;
      g[j] *= w[j];
    }
  };
  for (int c = threadIdx.x * 4; c < d; c += 4096) {
    get(c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a += g[j];
      b += g[j] * h[j];
    }
  }
  a = row_sum<1024>(a, s) / d;
  b = row_sum<1024>(b, s) / d;
  for (int c = threadIdx.x * 4; c < d; c += 4096) {
    get(c);
    float p[4] = {0.f, 0.f, 0.f, 0.f};
    if (past) load_some(past + r * ldp + c, d - c, p);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] += st.y * (g[j] - a - h[j] * b);
    store_some(dx + r * lddx + c, d - c, p);
  }
}
// A block has 256 columns of every `teams`-th row.  (Launched before dx is written: that may be in dy's place.)
template <typename T>
__global__ __launch_bounds__(256) void k_norm_back_cols(const float* dy, int64_t lddy, const T* x, int64_t ldx,
                                                        const float2* stats, const int32_t* n_rows, int64_t max_rows, int d,
                                                        int teams, float* part) {
  const int64_t rows = eff_count(max_rows, n_rows), cb = cdiv(d, 256), team = blockIdx.x / cb;
  const int64_t c = blockIdx.x % cb * 256 + threadIdx.x;
  if (c >= d) return;
  float dg = 0.f, db = 0.f;
  for (int64_t r = team; r < rows; r += teams) {
    const float g = dy[r * lddy + c];
    dg += g * ((Elem<T>::load(x, r * ldx + c) - stats[r].x) * stats[r].y);
    db += g;
  }
  part[team * 2 * d + c] = dg;
  part[team * 2 * d + d + c] = db;
}

// Columns of a row that a block keeps: 32 a thread of 1024; with the backward's five values to each, 16 a thread of 512.
constexpr int WIDE = 32768, WIDE_BACK = 8192;

// Teams of the backward: enough to fill the card, few enough that their shares of the sums over rows are few.  Rows that fit a
// wave have a wave each, 1,024 to 4,096 of them by the rows (backward and joining of 200,000 x 160 in float32: 209 us with
// 1,024, 124 with 2,048, 79 with 4,096, 80 with 8,192; of 7,997 x 445: 18.7, 15.7, 17.0 and 22.3), and four of them leave one share
// (forward and backward of 7,997 x 445 and 60,000 x 445 by waves 24.7 and 101, by blocks 27.7 and 138).  Wider ones have 1,024 blocks; with
// 256, 512, 1,024 and 2,048, forward and backward in bfloat16, us: 16,384 x 600 95, 61, 45 and 44; 16,384 x 2,048 190, 140, 103 and
// 114; 4,096 x 1,024 32, 25, 24 and 27; 4,096 x 4,096 72, 56, 63 and 70.  Where a block has a row or two of 4,096 and more, its shares
// outweigh them, and fewer blocks would be faster: 1,000 x 4,096 28, 27, 31 and 31; 1,000 x 8,192 35, 41, 52 and 52; 4,096 x
// 8,192 125, 131, 145 and 183.  Above 8,192 x and dy are read again for the sums over rows, by 64 teams (with 32, 64 and
// 256: 500 x 16,384 47, 49 and 58; 2,000 x 16,384 162, 169 and 181; 64 x 33,000 39, 44 and 43; 2,000 x 33,000 373, 363 and 379).
int back_teams(const mtgnn_norm_dims* d, int64_t rows) {
  if (d->d > WIDE_BACK) return (int)std::min<int64_t>(rows, 64);
  if (d->d > 512) return (int)std::min<int64_t>(rows, 1024);
  return (int)std::min<int64_t>(rows, std::min<int64_t>(std::max<int64_t>(rows / 4, 1024), 4096));
}
int back_shares(const mtgnn_norm_dims* d, int64_t rows) {
  const int teams = back_teams(d, rows);
  return d->d <= 512 ? (int)cdiv(teams, 4) : teams;
}

}  // namespace

int64_t norm_threads(const mtgnn_norm_dims* d) { return d->d <= 2048 ? 64 : d->d <= 8192 ? 256 : 1024; }   // (of many rows)
size_t norm_ws(const mtgnn_norm_dims* d, int64_t rows) { return (size_t)back_shares(d, rows) * 2 * d->d * 4; }

template <typename T>
mtgnn_status norm_t(const T* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const float* gamma, const float* beta,
                    const mtgnn_norm_dims* dims, T* y, int64_t ldy, float2* st, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const int d = dims->d;
  const float eps = dims->eps;
  const unsigned few = (unsigned)cdiv(max_rows, 4), all = (unsigned)max_rows;
  // A wave to a row, 32 elements a lane at most, where that leaves eight waves a CU (16,384 x 1,500 in bfloat16 25.4 us, by blocks 32.4;
  // 2,048 as wide 27.4 and 29.9); a block to one of few rows, in which less follows one after the other (the call takes as
  // long as its launch in both, 9.5 to 10 us up to 4,096 rows).
  const bool many = max_rows >= 2048;
  if (d <= 64 * V) k_norm<T, 64, 1><<<few, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (d <= 128 * V) k_norm<T, 64, 2><<<few, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (many && d <= 256 * V) k_norm<T, 64, 4><<<few, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (many && d <= 2048 && V == 4) k_norm<T, 64, 32 / V><<<few, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (d <= 256 * V) k_norm<T, 256, 1><<<all, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (d <= 512 * V) k_norm<T, 256, 2><<<all, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (d <= 8192) k_norm<T, 256, 32 / V><<<all, 256, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else if (d <= WIDE) k_norm<T, 1024, 32 / V><<<all, 1024, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  else k_norm_wide<T><<<all, 1024, 0, s>>>(x, ldx, n_rows, max_rows, gamma, beta, d, eps, y, ldy, st);
  MTGNN_CHECK_LAUNCH("layer_norm");
  return MTGNN_OK;
}

mtgnn_status norm_impl(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const float* gamma,
                       const float* beta, const mtgnn_norm_dims* d, void* y, int64_t ldy, float* stats, hipStream_t s) {
  if (d->dtype == MTGNN_BF16)
    return norm_t((const uint16_t*)x, ldx, n_rows, max_rows, gamma, beta, d, (uint16_t*)y, ldy, (float2*)stats, s);
  return norm_t((const float*)x, ldx, n_rows, max_rows, gamma, beta, d, (float*)y, ldy, (float2*)stats, s);
}

template <typename T>
mtgnn_status norm_bwd_t(const float* dy, int64_t lddy, const T* x, int64_t ldx, const float2* st, const int32_t* n_rows,
                        int64_t max_rows, const float* gamma, const float* past, int64_t ldp, const mtgnn_norm_dims* dims,
                        float* dx, int64_t lddx, float* dgamma, float* dbeta, float* ws, hipStream_t s) {
  const int d = dims->d, teams = back_teams(dims, max_rows);
  float* part = dgamma || dbeta ? ws : nullptr;
#define MTGNN_BACK(G, N)                                                                                               \
  k_norm_back<T, G, N><<<(unsigned)(G == 64 ? cdiv(teams, 4) : teams), G == 64 ? 256 : G, 0, s>>>(                     \
      dy, lddy, x, ldx, st, n_rows, max_rows, gamma, past, ldp, d, dx, lddx, teams, part)
  if (d <= 256) MTGNN_BACK(64, 1);
  else if (d <= 512) MTGNN_BACK(64, 2);
  else if (d <= 1024) MTGNN_BACK(256, 1);
  else if (d <= 2048) MTGNN_BACK(256, 2);
  else if (d <= 4096) MTGNN_BACK(256, 4);
  else if (d <= 8192) MTGNN_BACK(512, 4);
  else {
    if (part) k_norm_back_cols<T><<<(unsigned)(cdiv(d, 256) * teams), 256, 0, s>>>(dy, lddy, x, ldx, st, n_rows, max_rows, d, teams, part);
    MTGNN_CHECK_LAUNCH("layer_norm_back_cols");
    k_norm_back_wide<T><<<(unsigned)max_rows, 1024, 0, s>>>(dy, lddy, x, ldx, st, n_rows, max_rows, gamma, past, ldp, d, dx, lddx);
  }
#undef MTGNN_BACK
  MTGNN_CHECK_LAUNCH("layer_norm_back");
  if (part) {
    k_norm_join<<<(unsigned)cdiv(2 * d, 64), 512, 0, s>>>(part, back_shares(dims, max_rows), d, dgamma, dbeta);
    MTGNN_CHECK_LAUNCH("layer_norm_join");
  }
  return MTGNN_OK;
}

mtgnn_status norm_bwd_impl(const float* dy, int64_t lddy, const void* x, int64_t ldx, const float* stats,
                           const int32_t* n_rows, int64_t max_rows, const float* gamma, const float* past, int64_t ldp,
                           const mtgnn_norm_dims* d, float* dx, int64_t lddx, float* dgamma, float* dbeta, void* ws,
                           hipStream_t s) {
  if (d->dtype == MTGNN_BF16)
    return norm_bwd_t(dy, lddy, (const uint16_t*)x, ldx, (const float2*)stats, n_rows, max_rows, gamma, past, ldp, d, dx, lddx,
                      dgamma, dbeta, (float*)ws, s);
  return norm_bwd_t(dy, lddy, (const float*)x, ldx, (const float2*)stats, n_rows, max_rows, gamma, past, ldp, d, dx, lddx,
                    dgamma, dbeta, (float*)ws, s);
}

}  // namespace mtgnn
