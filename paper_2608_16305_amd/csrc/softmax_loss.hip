// Softmax cross entropy of each row's label over all classes, and its gradients, without the rows x classes logits:
//   l = x W^T + b,  loss_r = log sum_c exp l_rc - l_r,label,  loss = their mean over the rows with a label;
//   P = softmax(l) - [c is the row's label],  dx = P W,  dW = P^T x,  db = column sums of P, each times dloss / rows.
//
// The forward's product leaves per tile of columns each row's largest logit and the sum of exponentials relative to it; a row's
// are then joined.  The backward takes the classes in pieces: a piece's logits are formed again, become P in the workspace, and
// two products with W and x take it from there.  So 8 rows x classes x width operations are done where 6 are needed, and a
// piece of P, not all of it, is in memory.
//
// All products but those of few rows of float32 (k_loss_few) run on the bfloat16 matrix instructions with float32 sums.  bfloat16 x and
// W enter as they are.  Everything else enters as three bfloat16 parts, which hold 24 bits and float32's whole range (bf16_split.h):
// float32 x and W in the six products of parts that are not below 2^-24 of the whole, P in three with a bfloat16 operand.  (Two
// float16 parts of float32 operands and of P take three and two products.  But float16 lacks the range: elements below 2^-17 of
// a matrix's largest lost bits, a probability below 2^-39 was lost, and Adam divides a rare class's gradient by its own size.
// 8,192 x 32,768 x 1,024 in bfloat16 with gradients took 3,080 us with them for 3,980, 4,000 x 9,001 x 100 in float32 234 for 342.)
//
// Rows without a label are left out before anything is computed: the others' x is copied, row after row, padded with
// zeros to whole steps.
#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "ops.h"
#include "words.h"

namespace mtgnn {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int KS = 64;          // a step of the sums: 128 bytes of a line
constexpr int PAD = 64;         // rows and columns are padded to whole ones
constexpr int CHUNK = 1024;     // rows whose labels are counted together
constexpr int ROWS = 16;        // rows that a block copies
constexpr float LOG2E = 1.4426950408889634f;

__host__ __device__ inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// --------------------------------------------------------------------------- rows with a label

__device__ __forceinline__ bool has_label(const int32_t* label, int64_t r, int64_t rows, int n) {
  return r < rows && (uint32_t)label[r] < (uint32_t)n;
}

__device__ __forceinline__ int block_sum(int v, int* s) {   // over 256 threads
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0] + s[1] + s[2] + s[3];
  __syncthreads();
  return v;
}

// --------------------------------------------------------------------------- operands

// Eight elements of a row from c on (zeros from d on) in a padded matrix: as they are, or float32 in three parts.
template <typename T>
__device__ __forceinline__ void put_parts(const T* row, int c, int d, uint16_t* to, int64_t plane) {
  float v[8];
  uint32_t h[4], m[4], l[4];
  load_some(row + c, d - c, v);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = cvt2_bf16(v[2 * i], v[2 * i + 1]);
    *(uint4*)to = make_uint4(h[0], h[1], h[2], h[3]);
  } else {
    split_words<true>(v, h, m, l);
    *(uint4*)to = make_uint4(h[0], h[1], h[2], h[3]);
    *(uint4*)(to + plane) = make_uint4(m[0], m[1], m[2], m[3]);
    *(uint4*)(to + 2 * plane) = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// The forward's first launch: a block counts the labels of CHUNK rows.
__global__ __launch_bounds__(256) void k_loss_count(const int32_t* label, const int32_t* n_rows, int64_t max_rows, int n,
                                                    int32_t* counts) {
  __shared__ int s[4];
  const int64_t rows = eff_count(max_rows, n_rows);
  int v = 0;
#pragma unroll
  for (int u = 0; u < CHUNK / 256; ++u) v += has_label(label, (int64_t)blockIdx.x * CHUNK + u * 256 + threadIdx.x, rows, n);
  v = block_sum(v, s);
  if (threadIdx.x == 0) counts[blockIdx.x] = v;
}

// Rows of d as rows of dp: as they are, or in parts.  Block b.
template <typename T>
__device__ __forceinline__ void lay_table(const T* W, int64_t n, int d, int dp, uint16_t* to, int64_t plane, unsigned b) {
  const uint32_t units = dp / 8, e = b * 256 + threadIdx.x;
  const int64_t c = e / units;
  const int u = (int)(e % units) * 8;
  if (c < up(n, PAD)) put_parts<T>(W + c * d, u, c < n ? d : 0, to + c * dp + u, plane);   // (zeros behind the last)
}

// The forward's second launch (counts NULL: its only one, of so few rows that each block counts them).  Blocks below `blocks`:
// the rows with a label, one after the other: idx (which rows), lab, xc (their x,
// as it is or in parts; zeros behind the last one to a whole step); their number.  The last of
// them, past those of the rows, fill in the zeros.  The other blocks: W in parts, or padded.
template <typename T>
__global__ __launch_bounds__(256) void k_loss_lay(const T* x, int64_t ldx, const int32_t* label, const int32_t* n_rows,
                                                  int64_t max_rows, int n, int d, int dp, const int32_t* counts, int32_t* count,
                                                  int32_t* idx, int32_t* lab, uint16_t* xc, int64_t plane, float* row_loss,
                                                  unsigned blocks, const T* W, uint16_t* table) {
  constexpr int PARTS = sizeof(T) == 2 ? 1 : 3;
  __shared__ int s[4], src[ROWS];
  if (blockIdx.x >= blocks) {
    lay_table<T>(W, n, d, dp, table, up(n, PAD) * dp, blockIdx.x - blocks);
    return;
  }
  const int64_t rows = eff_count(max_rows, n_rows), r0 = (int64_t)blockIdx.x * ROWS;
  const int chunks = (int)cdiv(max_rows, CHUNK), units = dp / 8;
  const bool behind = r0 >= max_rows;
  const int mine = behind ? chunks : (int)(r0 / CHUNK);
  int v = 0;
  for (int i = threadIdx.x; counts && i < mine; i += 256) v += counts[i];
  for (int64_t r = (counts ? (int64_t)mine * CHUNK : 0) + threadIdx.x; r < min(r0, max_rows); r += 256)
    v += has_label(label, r, rows, n);
  const int first = block_sum(v, s);
  if (behind) {
    const int j0 = (int)(r0 - up(max_rows, ROWS));
    if (j0 == 0 && threadIdx.x == 0) *count = first;
    const int64_t end = up(first, PAD);
    for (int e = threadIdx.x; e < ROWS * units; e += 256) {
      const int64_t r = first + j0 + e / units;
      if (r >= end) break;
#pragma unroll
      for (int q = 0; q < PARTS; ++q) *(uint4*)(xc + q * plane + r * dp + e % units * 8) = make_uint4(0u, 0u, 0u, 0u);
    }
    return;
  }
  int here = 0;
  if (threadIdx.x < 64) {
    const int64_t r = r0 + threadIdx.x;
    const bool ok = threadIdx.x < ROWS && has_label(label, r, rows, n);
    const uint64_t have = __ballot(ok);
    const int at = __popcll(have & ((uint64_t(1) << threadIdx.x) - 1));
    here = __popcll(have);
    if (ok) {
      src[at] = (int)threadIdx.x;
      idx[first + at] = (int32_t)r;
      lab[first + at] = label[r];
    } else if (threadIdx.x < ROWS && r < rows && row_loss) {
      row_loss[r] = 0.f;
    }
    if (threadIdx.x == 0) s[0] = here;
  }
  __syncthreads();
  here = s[0];
  for (int e = threadIdx.x; e < here * units; e += 256) {
    const int k = e / units, c = e % units * 8;
    put_parts<T>(x + (r0 + src[k]) * ldx, c, d, xc + (int64_t)(first + k) * dp + c, plane);
  }
}

// The backward's first launch: zeros in dx of the rows without a label (zero_blocks); W in parts or padded, or the rows behind the last
// whole step of one that is used in place (table_blocks: `wn` rows from W on, `wdp` apart); x's rows where the forward has
// left them in float32.
template <typename T>
__global__ __launch_bounds__(256) void k_loss_back_lay(const int32_t* label, const int32_t* n_rows, int64_t max_rows, int n, int d,
                                                       float* dx, int64_t lddx, unsigned zero_blocks, const T* W, int64_t wn,
                                                       int wdp, uint16_t* table, unsigned table_blocks, const T* xc, int64_t Rp, int dp,
                                                       uint16_t* xh) {
  if (blockIdx.x >= zero_blocks + table_blocks) {
    lay_table<T>(xc, Rp, dp, dp, xh, Rp * dp, blockIdx.x - zero_blocks - table_blocks);
    return;
  }
  if (blockIdx.x >= zero_blocks) {
    lay_table<T>(W, wn, d, wdp, table, up(wn, PAD) * wdp, blockIdx.x - zero_blocks);
    return;
  }
  const uint32_t dv = (uint32_t)cdiv(d, 4), e = blockIdx.x * 256 + threadIdx.x;
  const int64_t r = e / dv;
  const int c = (int)(e % dv) * 4;
  if (r >= eff_count(max_rows, n_rows) || (uint32_t)label[r] < (uint32_t)n) return;
  const float z[4] = {0.f, 0.f, 0.f, 0.f};
  store_some(dx + r * lddx + c, d - c, z);
}

// --------------------------------------------------------------------------- the products

enum { STAT, PROB, DX, DW };

// What P is multiplied by in the gradients: 1 / rows, times the loss's own gradient.
__device__ __forceinline__ float loss_scale(int64_t rows, const float* dloss) {
  return rows > 0 ? (dloss ? *dloss : 1.f) / (float)rows : 0.f;
}

struct Prod {
  const uint16_t *A, *B;         // A: the result's rows, B: its columns
  int64_t lda, ldb, planeA, planeB;
  uint32_t codeA, codeB;         // the parts of each segment, two bits each
  int segs, split;               // split: blocks that share a tile's sum, each leaving its own in `out`
  int64_t rows, cols, K;         // the most rows; K: of a segment (its last step has a k that may be read)
  int64_t dimA, dimB;            // elements of a line across the sum that may be read
  int64_t endB;                  // k of B that may be read, where a W in place may end inside a step (STAT, PROB, DX)
  int64_t tail;                  // DX: where that step's rows are, and zeros behind them, from B on
  int64_t tr, tc;                // tiles
  const int32_t* count;          // rows with a label: bounds the rows (STAT, PROB, DX) or K (DW)
  // epilogue
  const float* b;                // of the first column on
  const int32_t *lab, *idx;
  int64_t c0;                    // first column's class
  float2* part;                  // STAT: [tc][ld_part]
  int64_t ld_part;
  float* at_label;
  const float2* stat;            // PROB: largest logit, 1 / sum
  uint16_t* P;                   // three parts
  int64_t ldp, planeP;
  float* cols_part;              // column sums of P, of each half tile's rows, or NULL
  float* out;
  int64_t ldo;
  const float* dloss;
  int add;
};

// Lines go straight to LDS, 16 bytes a lane.  Along the sum: a line's eight units are swizzled by the line, as in
// linear.hip.  Across it: a k's 32-byte units by k, and the transposing read of 4 k x 16 columns gives a lane its four k;
// the 16 lanes of such a read, and their neighbours, meet every bank once.
// An operand's T lines of a step, loaded by NW waves; its lines are contiguous along the sum (ALONG) or across it.
template <bool ALONG, int T, int NW>
struct Lines {
  static constexpr int WORDS = T * KS / 2, LOADS = T * KS / 512 / NW;   // in LDS; a wave's loads
  static constexpr int UNITS = T / 8;                                   // 16-byte units of a k
  static_assert(LOADS >= 1, "every wave loads");
  typedef __attribute__((address_space(3))) void* lds_ptr;
  typedef __attribute__((address_space(3))) s16x4* lds_tr;

  // The k of a step of a lane's load i.
  __device__ __forceinline__ static int k_of(int wid, int lane, int i) {
    return ALONG ? 8 * ((lane & 7) ^ (lane >> 3)) : (LOADS * wid + i) * (64 / UNITS) + lane / UNITS;
  }
  // This wave's loads: bytes from the tile's first line at a step's first k.  (Below 2^32: 256 lines of 2^22 elements, or 32 of
  // them.)
  __device__ __forceinline__ static void sources(int64_t ld, int64_t lines, int64_t dim, int wid, int lane, uint32_t (&off)[LOADS]) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int k = k_of(wid, lane, i);
      if constexpr (ALONG) {
        const int row = 8 * (LOADS * wid + i) + (lane >> 3);
        off[i] = 2u * ((uint32_t)min((int64_t)row, lines - 1) * (uint32_t)ld + k);
      } else {
        const int q = lane % UNITS, col = ((q >> 1 ^ ((k & 3) | (k >> 3 & 1) << 2)) * 2 + (q & 1)) * 8;
        off[i] = 2u * ((uint32_t)k * (uint32_t)ld + (uint32_t)min((int64_t)col, dim - 8));
      }
    }
  }
  // Load i of a step that starts at `p`.  `left`: how many of its k may be read; the lanes past them read the step's first (it meets
  // zeros of the other operand).
  template <bool END>
  __device__ __forceinline__ static void load(uint32_t* buf, const uint16_t* p, const uint32_t (&off)[LOADS], int64_t left, int wid,
                                              int lane, int i) {
    uint32_t o = off[i];
    if (END && left < KS) {
      const int k = k_of(wid, lane, i);
      if (k >= left) o -= 2u * (uint32_t)k;
    }
    __builtin_amdgcn_global_load_lds((void*)((const char*)p + o), (lds_ptr)(buf + (LOADS * wid + i) * 256), 16, 0, 0);
  }
  // A lane's byte for the lines from l0 (a multiple of 64) on, and what is read there of the 16 lines from l0 + 16 l, half kk.
  __device__ __forceinline__ static uint32_t place(int l0, int fr, int fg) {
    if (ALONG) return (l0 + fr) * (2 * KS) + (fg ^ (fr & 7)) * 16;
    return ((8 * fg + (fr >> 2)) * (2 * T) + ((fr >> 2) | (fg & 1) << 2) * 32 + (fr & 3) * 8) ^ 2 * l0;
  }
  __device__ __forceinline__ static bf16x8_t frag(uint32_t* buf, uint32_t at, int l, int kk) {
    if constexpr (ALONG) {
      return __builtin_bit_cast(bf16x8_t, *(const uint4*)((char*)buf + ((at ^ 64 * kk) + l * 16 * 2 * KS)));
    } else {
      char* a = (char*)buf + ((at ^ 32 * l) + kk * 32 * 2 * T);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)a);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(a + 4 * 2 * T));
      return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Blocks run on the 8 XCDs in turn, each with its own L2: a contiguous eighth of the tiles to each, in groups of eight tiles of
// rows by all of columns, so that the blocks that run together share lines of both operands.
__device__ __forceinline__ void my_tile(const Prod& p, int64_t& tr, int64_t& tc, int& share) {
  const int64_t L = blockIdx.x, n = p.tr * p.tc * p.split, full = n & ~int64_t(7);
  int64_t V = L < full ? (L & 7) * (full >> 3) + (L >> 3) : L;
  share = (int)(V / (p.tr * p.tc));
  V %= p.tr * p.tc;
  constexpr int64_t G = 8;
  const int64_t group = V / (G * p.tc), in = V % (G * p.tc), h = min(G, p.tr - group * G);
  tr = group * G + in % h;
  tc = in / h;
}

__device__ __forceinline__ f32x4 mma(bf16x8_t a, bf16x8_t b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// TR x TC tiles, a wave has 16 WR x 64 of one: all of its rows where they are 64, else half of them.
template <int TR, int TC>
struct Shape {
  static constexpr int WCOLS = TC / 64, WROWS = TR == 64 ? 1 : 2, NW = WROWS * WCOLS;
  static constexpr int WR = TR / 16 / WROWS, WC = 4, LINES = TR, COLUMNS = TC;
};

// What exponentials are relative to, where m is the largest logit: m, but not an infinite one, whose difference from itself is NaN.
// Nothing but classes of logit -inf have a sum of zeros so, and one of +inf an infinite sum, in which a NaN still shows.
__device__ __forceinline__ float base_of(float m) { return fabsf(m) < INFINITY ? m : 0.f; }

// Joins (largest, sum of exponentials relative to it).
__device__ __forceinline__ void join(float2& q, float2 o) {
  const float m = fmaxf(q.x, o.x), from = base_of(m);
  q.y = q.y * __builtin_amdgcn_exp2f((q.x - from) * LOG2E) + o.y * __builtin_amdgcn_exp2f((o.x - from) * LOG2E);
  q.x = m;
}

// What the end of a tile needs of its rows and columns, requested before the products so that it need not be waited for.
template <int KIND, class S>
struct Ahead {
  int at[S::WR];         // the label's place in the lane's columns
  float b[S::WC][4];
  __device__ __forceinline__ void load(const Prod& p, int64_t ra, int64_t ca, int64_t rows) {
    if constexpr (KIND == STAT || KIND == PROB) {
#pragma unroll
      for (int i = 0; i < S::WR; ++i) {
        const int64_t r = min(ra + 16 * i, rows - 1);
        at[i] = p.lab[r];
      }
#pragma unroll
      for (int j = 0; j < S::WC; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) b[j][e] = 0.f;
        if (p.b) load_some(p.b + ca + 16 * j, (int)max((int64_t)0, min((int64_t)4, p.cols - ca - 16 * j)), b[j]);
      }
    }
  }
};

// What becomes of a wave's sums.  FULL: the tile has all of its columns.  s: LDS that nothing uses any more.
template <int KIND, class S, bool FULL, int WR, int WC>
__device__ __forceinline__ void leave(const Prod& p, f32x4 (&acc)[WR][WC], Ahead<KIND, S>& h, uint32_t* lds, int64_t r0, int64_t c0,
                                      int64_t rows, int64_t count, int share, int wid, int lane) {
  const int wr = wid / S::WCOLS * (16 * WR), wc = wid % S::WCOLS * 64, fr = lane & 15, fg = lane >> 4;
  const int64_t ca = c0 + wc + 4 * fg, ra = r0 + wr + fr;
  auto &at = h.at;
  float2 st[WR];         // the row's largest logit, 1 / sum
  if constexpr (KIND == STAT || KIND == PROB) {
#pragma unroll
    for (int i = 0; i < WR; ++i) {
      const bool live = ra + 16 * i < rows;
      at[i] = live ? (int)(at[i] - p.c0 - ca) : -1;
      if (KIND == PROB) st[i] = live ? p.stat[ra + 16 * i] : make_float2(INFINITY, 0.f);   // behind the last row: exponentials of -inf
    }
#pragma unroll
    for (int j = 0; j < WC; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < WR; ++i) {
          acc[i][j][e] += h.b[j][e];
          if (!FULL && ca + 16 * j + e >= p.cols) acc[i][j][e] = -INFINITY;
        }
  }
  // (a row's label is in one of the waves' columns: in most there is none)
  const auto has = [&](int i) { return __any((unsigned)at[i] < 64u && (at[i] & 15) < 4); };
  if constexpr (KIND == STAT) {
    float2* s = (float2*)lds;   // [columns' waves][lines]
#pragma unroll
    for (int i = 0; i < WR; ++i) {
      float m = -INFINITY, v = 0.f;
#pragma unroll
      for (int j = 0; j < WC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
      if (has(i)) {
#pragma unroll
        for (int j = 0; j < WC; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at[i] == 16 * j + e) p.at_label[ra + 16 * i] = acc[i][j][e];
      }
      m = fmaxf(m, __shfl_xor(m, 16, 64));
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      const float from = base_of(m);
#pragma unroll
      for (int j = 0; j < WC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v += __builtin_amdgcn_exp2f((acc[i][j][e] - from) * LOG2E);
      v += __shfl_xor(v, 16, 64);
      v += __shfl_xor(v, 32, 64);
      if (fg == 0) s[wid % S::WCOLS * S::LINES + wr + 16 * i + fr] = make_float2(m, v);
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= S::LINES || r0 + t >= rows) return;
    float2 q = s[t];
#pragma unroll
    for (int w = 1; w < S::WCOLS; ++w) join(q, s[w * S::LINES + t]);
    p.part[c0 / S::COLUMNS * p.ld_part + r0 + t] = q;
  }
  if constexpr (KIND == PROB) {
    float sum[WC][4];
#pragma unroll
    for (int j = 0; j < WC; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[j][e] = 0.f;
    const int64_t end = up(rows, PAD);   // zeros in the rows behind the last, to a whole step
#pragma unroll
    for (int i = 0; i < WR; ++i) {
#pragma unroll
      for (int j = 0; j < WC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_amdgcn_exp2f((acc[i][j][e] - st[i].x) * LOG2E) * st[i].y;
      if (has(i)) {
#pragma unroll
        for (int j = 0; j < WC; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at[i] == 16 * j + e) acc[i][j][e] -= 1.f;
      }
      if (p.cols_part) {
#pragma unroll
        for (int j = 0; j < WC; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[j][e] += acc[i][j][e];
      }
      // sixteen rows through LDS (the wave's own place): written as they lie there, in whole 128 bytes (in the lanes'
      // order 32 bytes a row at a time P in two parts took 823 us for 612, 7,373 x 32,768 x 1,024)
      char* w = (char*)lds + wid * (3 * 16 * 144);
#pragma unroll
      for (int j = 0; j < WC; ++j) {
        const f32x4 v = acc[i][j];
        char* to = w + fr * 144 + 32 * j + 8 * fg;
        const uint2 hi = make_uint2(cvt2_bf16(v[0], v[1]), cvt2_bf16(v[2], v[3]));
        const float a[4] = {v[0] - lo_bf16(hi.x), v[1] - hi_bf16(hi.x), v[2] - lo_bf16(hi.y), v[3] - hi_bf16(hi.y)};
        const uint2 mid = make_uint2(cvt2_bf16(a[0], a[1]), cvt2_bf16(a[2], a[3]));
        *(uint2*)to = hi;
        *(uint2*)(to + 16 * 144) = mid;
        *(uint2*)(to + 2 * 16 * 144) = make_uint2(cvt2_bf16(a[0] - lo_bf16(mid.x), a[1] - hi_bf16(mid.x)),
                                                  cvt2_bf16(a[2] - lo_bf16(mid.y), a[3] - hi_bf16(mid.y)));
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int h8 = 0; h8 < 2; ++h8) {
          const int line = 8 * h8 + (lane >> 3);
          const uint4 v = *(const uint4*)(w + q * 16 * 144 + line * 144 + (lane & 7) * 16);
          const int64_t rr = r0 + wr + 16 * i + line, cc = c0 + wc + (lane & 7) * 8;
          if (rr < end && (FULL || cc < p.ldp)) *(uint4*)(p.P + q * p.planeP + rr * p.ldp + cc) = v;
        }
      __builtin_amdgcn_wave_barrier();
    }
    if (p.cols_part) {
#pragma unroll
      for (int j = 0; j < WC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) sum[j][e] += __shfl_xor(sum[j][e], o, 64);
        }
      if (fr == 0 && r0 + wr < rows)
#pragma unroll
        for (int j = 0; j < WC; ++j)
          if (FULL || ca + 16 * j < p.ldp)
            *(float4*)(p.cols_part + (r0 + wr) / (16 * WR) * p.ldp + ca + 16 * j) =
                make_float4(sum[j][0], sum[j][1], sum[j][2], sum[j][3]);
    }
  }
  if constexpr (KIND == DX || KIND == DW) {
    const bool whole = p.split == 1;   // else the sums as they are, for k_loss_shares
    const float scale = whole ? loss_scale(count, p.dloss) : 1.f;
    float* const out = p.out + (whole ? 0 : share * p.rows * p.ldo);
    const bool add = KIND == DX && whole && p.add;
    float* w = (float*)lds + wid * (16 * 68);   // (as above: whole 256 bytes of a row)
#pragma unroll
    for (int i = 0; i < WR; ++i) {
#pragma unroll
      for (int j = 0; j < WC; ++j) *(f32x4*)(w + fr * 68 + 16 * j + 4 * fg) = acc[i][j];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int line = 4 * q + fg;
        const f32x4 f = *(const f32x4*)(w + line * 68 + 4 * fr);
        const int64_t r = r0 + wr + 16 * i + line, c = c0 + wc + 4 * fr;
        const int n = FULL ? 4 : (int)min((int64_t)4, p.cols - c);
        if (r >= rows || n <= 0) continue;
        float* o = out + (KIND == DX && whole ? (int64_t)p.idx[r] : r) * p.ldo + c;
        float v[4], old[4] = {0.f, 0.f, 0.f, 0.f};
        if (add) load_some(o, n, old);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = f[e] * scale + old[e];
        store_some(o, n, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <int KIND, int TR, int TC>
__global__ __launch_bounds__(TR == 256 ? 512 : 256, 2) void k_loss_product(Prod p) {
  using S = Shape<TR, TC>;
  constexpr bool AK = KIND != DW, BK = KIND == STAT || KIND == PROB;
  constexpr int WR = S::WR, WC = S::WC;
  using LA = Lines<AK, TR, S::NW>;
  using LB = Lines<BK, TC, S::NW>;
  constexpr int WORDS = LA::WORDS + LB::WORDS, LOADS = LA::LOADS + LB::LOADS;
  __shared__ __align__(1024) uint32_t buf0[WORDS], buf1[WORDS];
  int64_t tr, tc;
  int share;
  my_tile(p, tr, tc, share);
  const int64_t count = *p.count, rows = KIND == DW ? p.rows : min(p.rows, count);
  const int64_t K = KIND == DW ? up(count, PAD) : p.K;
  const int64_t r0 = tr * TR, c0 = tc * TC;
  if (r0 >= rows) return;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wid / S::WCOLS * (16 * WR), wc = wid % S::WCOLS * 64, fr = lane & 15, fg = lane >> 4;
  uint32_t offA[LA::LOADS], offB[LB::LOADS];
  LA::sources(p.lda, rows - r0, p.dimA - (AK ? 0 : r0), wid, lane, offA);
  LB::sources(p.ldb, p.cols - c0, p.dimB - (BK ? 0 : c0), wid, lane, offB);
  const uint16_t *fromA = p.A + r0 * (AK ? p.lda : 1), *fromB = p.B + c0 * (BK ? p.ldb : 1);
  Ahead<KIND, S> ahead;
  ahead.load(p, r0 + wr + fr, c0 + wc + 4 * fg, rows);
  f32x4 acc[WR][WC];
#pragma unroll
  for (int i = 0; i < WR; ++i)
#pragma unroll
    for (int j = 0; j < WC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int per = (int)cdiv(K, KS), all = per * p.segs, each = (all + p.split - 1) / p.split;
  const int steps = max(0, min(each, all - share * each));
  int seg = steps > 0 ? share * each / per : 0, k = share * each - seg * per;   // of the next step to load
  int at = 0;
  // Where B's step from k0 on is.  (The choice by masks: by a branch or a select it took vector registers that the sums need.)
  const auto of_b = [&](int64_t k0) __attribute__((always_inline)) {
    const int64_t o = (p.codeB >> 2 * seg & 3) * p.planeB + k0 * (BK ? 1 : p.ldb), past = (p.endB - KS - k0) >> 63;
    return KIND == DX ? o ^ ((o ^ p.tail) & past) : o;
  };
  const auto load = [&](uint32_t* buf, int u) __attribute__((always_inline)) {
    const int64_t k0 = (int64_t)k * KS;
    if (u < LA::LOADS)
      LA::template load<false>(buf, fromA + (p.codeA >> 2 * seg & 3) * p.planeA + k0 * (AK ? 1 : p.lda), offA, KS, wid, lane, u);
    else
      LB::template load<BK>(buf + LA::WORDS, fromB + of_b(k0), offB, p.endB - k0, wid, lane, u - LA::LOADS);
    if (u + 1 < LOADS) return;
    const int go = ++at < steps, turn = k + 1 == per;   // (the last step's again past it)
    seg += go & turn;
    k = go ? (turn ? 0 : k + 1) : k;
  };
  uint32_t atA = LA::place(wr, fr, fg), atB = LB::place(wc, fr, fg);
  // This wave's loads have arrived and its reads are done, then everybody's.
  const auto ready = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // A step is 2 WR groups of WC matrix instructions, a line of A by all of the wave's B; a line is read LOOK groups before it is
  // used, the B of a half step in the half step before.  WR / 2 groups before the end, and a group after the step's last reads, every
  // wave has read the whole step and the next one has arrived: the next one's operands are read, and the buffer is filled with the
  // step after it.  What is behind the barrier for a wave to do at once are matrix instructions.  (Past the last step loads and
  // reads go on, without a branch, and what they bring is not used.)  The buffers are two objects, so that the compiler knows that
  // reads of one do not wait for the loads into the other.
  constexpr int GROUPS = 2 * WR, READY = GROUPS - WR / 2, LOOK = WR / 2 + 1;
  bf16x8_t a[WR], b[2][WC];
  const auto work = [&](uint32_t* buf, uint32_t* next) __attribute__((always_inline)) {
    // (places formed again each time: kept for every line, they would not leave the sums their registers)
    asm volatile("" : "+v"(atA), "+v"(atB));
#pragma unroll
    for (int m = 0; m < GROUPS; ++m) {
      if (m == READY) ready();
#pragma unroll
      for (int j = 0; j < WC; ++j) acc[m % WR][j] = mma(b[m / WR][j], a[m % WR], acc[m % WR][j]);
      __builtin_amdgcn_sched_barrier(0);
      if (m >= READY) {
        constexpr int PER = LOADS / (WR / 2);
#pragma unroll
        for (int u = 0; u < PER; ++u) load(buf, (m - READY) * PER + u);
      }
      const int q = m + LOOK;   // line of this step, or (from READY on, two of them at first) of the next
      if (q < GROUPS) a[q % WR] = LA::frag(buf, atA, q % WR, q / WR);
      if (m == READY) a[0] = LA::frag(next, atA, 0, 0);
      if (m >= READY) a[m - READY + 1] = LA::frag(next, atA, m - READY + 1, 0);
      const int half = m < WR / 2 ? 1 : 0, first = half ? m : m - READY;
      if (half || m >= READY) {
#pragma unroll
        for (int j = first * 2 * WC / WR; j < (first + 1) * 2 * WC / WR; ++j) b[half][j] = LB::frag((half ? buf : next) + LA::WORDS, atB, j, half);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  static_assert(LOADS % (WR / 2) == 0 && 2 * WC % WR == 0, "loads and reads of B of a group");
  if (steps > 0) {
    // Two steps at a time (one way out of the loop, so that the sums stay where they are): an odd number has zeros before the first.
    const bool zeros = steps & 1;
    for (int i = threadIdx.x; zeros && i < WORDS; i += 64 * S::NW) buf0[i] = 0u;
    if (!zeros)
#pragma unroll
      for (int u = 0; u < LOADS; ++u) load(buf0, u);
    ready();
#pragma unroll
    for (int u = 0; u < LOADS; ++u) load(buf1, u);
#pragma unroll
    for (int i = 0; i < LOOK; ++i) a[i] = LA::frag(buf0, atA, i, 0);
#pragma unroll
    for (int j = 0; j < WC; ++j) b[0][j] = LB::frag(buf0 + LA::WORDS, atB, j, 0);
    for (int step = 0; step < steps; step += 2) {
      work(buf0, buf1);
      work(buf1, buf0);
    }
  }
  __syncthreads();   // (waits for the loads and reads that nothing used)

  // A lane has columns c0 + wc + 16 j + 4 fg .. + 3 of the rows r0 + wr + 16 i + fr.  Most tiles have all of their columns, and
  // no test of each.
  if (c0 + TC <= p.cols) leave<KIND, S, true>(p, acc, ahead, buf0, r0, c0, rows, count, share, wid, lane);
  else leave<KIND, S, false>(p, acc, ahead, buf0, r0, c0, rows, count, share, wid, lane);
}

// --------------------------------------------------------------------------- few rows of float32

// For few rows every product is reading W or writing dW.  Those of float32 take W as it is, on the float32 matrix instructions (256
// operations a cycle of a compute unit: 64 rows take about as long as the reading, 16 a quarter); in parts it is
// laid out and read (14 x 142,281 x 1,024 forward 665 us for 130).  A block has 64 CF classes and up to 64 rows; a
// lane reads 16 bytes of a class at a k four apart from its neighbours', and x, through LDS, in the same order, so that the
// fragments need no more than that.  The forward leaves what STAT does, and x's rows with a label as they are; the backward
// forms the logits again, leaves P [classes][16 RF] for dx, and writes db and, from P and x in LDS, dW.
struct Few {
  const float *x, *W, *b;
  int64_t ldx;
  const int32_t *label, *n_rows;
  int64_t max_rows;
  int n, d;
  int32_t *count, *idx, *lab;
  float* xc;                // x's rows with a label, dp apart, zeros behind d; the forward's may be NULL
  int dp;
  float2* part;             // forward
  int64_t ld_part;
  float *at_label, *row_loss;
  const float2* stat;       // backward
  const float* dloss;
  float *P, *db, *dW;       // each or NULL
  int groups;               // of 64 rows: blocks that follow each other have a tile's
};
constexpr int FEW = 256, KC = 64, LDC = KC + 4;
template <int RF, int CF, bool BACK>
__global__ __launch_bounds__(256) void k_loss_few(Few p) {
  __shared__ __align__(16) float xs[2][16 * RF][LDC];
  __shared__ __align__(16) float ps[BACK ? 64 * CF : 1][16 * RF + 4], out[BACK ? 4 : 1][16][LDC];
  __shared__ int src[16 * RF], lab[16 * RF], in_wave[4];
  __shared__ float2 st[4][16 * RF];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, fr = lane & 15, fg = lane >> 4;
  const int tile = blockIdx.x / p.groups, group = blockIdx.x % p.groups, r0 = group * 16 * RF;
  const int c0 = tile * 64 * CF + wid * 16 * CF, steps = (int)cdiv(p.d, KC);
  // the first step of W and the bias do not wait for the labels
  const float* w[CF];
#pragma unroll
  for (int j = 0; j < CF; ++j) w[j] = p.W + (int64_t)min(c0 + 16 * j + fr, p.n - 1) * p.d + 4 * fg;
  float wv[CF][4][4], bias[CF][4];
  const auto load_w = [&](int k) __attribute__((always_inline)) {
    const bool whole = k + KC <= p.d;
#pragma unroll
    for (int j = 0; j < CF; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t) load_some(w[j] + k + 16 * t, whole ? 4 : p.d - k - 16 * t - 4 * fg, wv[j][t]);
  };
  load_w(0);
#pragma unroll
  for (int j = 0; j < CF; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[j][e] = p.b ? p.b[min(c0 + 16 * j + 4 * fg + e, p.n - 1)] : 0.f;

  int all = 0;
  if constexpr (BACK) {
    all = *p.count;
    if (threadIdx.x < all) lab[threadIdx.x] = p.lab[threadIdx.x];
  } else {
    const int64_t rows = eff_count(p.max_rows, p.n_rows);
    const int t = threadIdx.x;
    const bool ok = has_label(p.label, t, rows, p.n);
    const uint64_t have = __ballot(ok);
    if (lane == 0) in_wave[wid] = __popcll(have);
    __syncthreads();
    int at = __popcll(have & ((uint64_t(1) << lane) - 1));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      at += w < wid ? in_wave[w] : 0;
      all += in_wave[w];
    }
    const int here = at - r0;
    if (ok && here >= 0 && here < 16 * RF) src[here] = t, lab[here] = p.label[t];
    if (blockIdx.x == 0) {
      if (t == 0) *p.count = all;
      if (ok) p.idx[at] = t, p.lab[at] = p.label[t];
      else if (t < rows && p.row_loss) p.row_loss[t] = 0.f;
    }
  }
  const int count = min(all - r0, 16 * RF);   // rows of the group
  if (!BACK && count <= 0) return;
  __syncthreads();

  const int xl = threadIdx.x >> 4, xk = 4 * (threadIdx.x & 15);
  const float* xr[RF];
#pragma unroll
  for (int u = 0; u < RF; ++u) {
    const int r = 16 * u + xl;
    if constexpr (BACK) xr[u] = r < count ? p.xc + (int64_t)r * p.dp + xk : nullptr;
    else xr[u] = r < count ? p.x + (int64_t)src[r] * p.ldx + xk : nullptr;
  }
  float xv[RF][4];
  const auto load_x = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < RF; ++u)
      if (!xr[u]) xv[u][0] = xv[u][1] = xv[u][2] = xv[u][3] = 0.f;
      else load_some(xr[u] + k, BACK || k + KC <= p.d ? 4 : p.d - k - xk, xv[u]);
  };
  const auto put_x = [&](float (*xb)[LDC]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < RF; ++u) *(float4*)&xb[16 * u + xl][xk] = make_float4(xv[u][0], xv[u][1], xv[u][2], xv[u][3]);
  };
  f32x4 acc[RF][CF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < CF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  load_x(0);
  for (int step = 0; step < steps; ++step) {
    float (*xb)[LDC] = xs[step & 1];
    float now[CF][4][4];
#pragma unroll
    for (int j = 0; j < CF; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) now[j][t][e] = wv[j][t][e];
    put_x(xb);
    if (!BACK && p.xc && tile == 0) {
#pragma unroll
      for (int u = 0; u < RF; ++u)
        *(float4*)(p.xc + (int64_t)(r0 + 16 * u + xl) * p.dp + step * KC + xk) = make_float4(xv[u][0], xv[u][1], xv[u][2], xv[u][3]);
    }
    if (step + 1 < steps) {
      load_w((step + 1) * KC);
      load_x((step + 1) * KC);
    }
    __syncthreads();   // (every wave has read what the step before last left here)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 f[RF];
#pragma unroll
      for (int i = 0; i < RF; ++i) f[i] = *(const f32x4*)&xb[16 * i + fr][16 * t + 4 * fg];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < CF; ++j)
#pragma unroll
          for (int i = 0; i < RF; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(now[j][t][e], f[i][e], acc[i][j], 0, 0, 0);
    }
  }

  // A lane has classes c0 + 16 j + 4 fg .. + 3 of the rows 16 i + fr.
  if constexpr (!BACK) {
#pragma unroll
    for (int i = 0; i < RF; ++i) {
      const int r = 16 * i + fr, at = r < count ? lab[r] : -1;
      float m = -INFINITY, v = 0.f;
#pragma unroll
      for (int j = 0; j < CF; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = c0 + 16 * j + 4 * fg + e;
          const float l = c < p.n ? acc[i][j][e] + bias[j][e] : -INFINITY;
          acc[i][j][e] = l;
          if (c == at) p.at_label[r0 + r] = l;
          m = fmaxf(m, l);
        }
      m = fmaxf(m, __shfl_xor(m, 16, 64));
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      const float from = base_of(m);
#pragma unroll
      for (int j = 0; j < CF; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v += __builtin_amdgcn_exp2f((acc[i][j][e] - from) * LOG2E);
      v += __shfl_xor(v, 16, 64);
      v += __shfl_xor(v, 32, 64);
      if (fg == 0) st[wid][r] = make_float2(m, v);
    }
    __syncthreads();
    const int r = threadIdx.x;
    if (r >= count) return;
    float2 q = st[0][r];
#pragma unroll
    for (int k = 1; k < 4; ++k) join(q, st[k][r]);
    p.part[tile * p.ld_part + r0 + r] = q;
  } else {
    const float scale = loss_scale(count, p.dloss);
    float sum[CF][4];
#pragma unroll
    for (int i = 0; i < RF; ++i) {
      const int r = 16 * i + fr, at = r < count ? lab[r] : -1;
      const float2 s = r < count ? p.stat[r] : make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < CF; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = c0 + 16 * j + 4 * fg + e;
          float v = __builtin_amdgcn_exp2f((acc[i][j][e] + bias[j][e] - s.x) * LOG2E) * s.y;
          if (c == at) v -= 1.f;
          if (r >= count) v = 0.f;
          sum[j][e] = i ? sum[j][e] + v : v;
          if (p.P && c < p.n) p.P[(int64_t)c * (16 * RF) + r] = v;
          ps[wid * 16 * CF + 16 * j + 4 * fg + e][r] = v;
        }
      }
    }
    if (p.db) {
#pragma unroll
      for (int j = 0; j < CF; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) sum[j][e] += __shfl_xor(sum[j][e], o, 64);
          const int c = c0 + 16 * j + 4 * fg + e;
          if (fr == 0 && c < p.n) p.db[c] = sum[j][e] * scale;
        }
    }
    if (!p.dW) return;
    // dW of the wave's classes, 64 k at a time: P's rows, and x's, four apart in a lane; out through LDS in whole 256 bytes.
    f32x4 pf[CF][RF];
    __syncthreads();   // (of xs too)
#pragma unroll
    for (int j = 0; j < CF; ++j)
#pragma unroll
      for (int t = 0; t < RF; ++t) pf[j][t] = *(const f32x4*)&ps[wid * 16 * CF + 16 * j + fr][16 * t + 4 * fg];
    load_x(0);
    for (int step = 0; step < steps; ++step) {
      float (*xb)[LDC] = xs[step & 1];
      put_x(xb);
      if (step + 1 < steps) load_x((step + 1) * KC);
      __syncthreads();
      f32x4 g[CF][4];
#pragma unroll
      for (int j = 0; j < CF; ++j)
#pragma unroll
        for (int h = 0; h < 4; ++h) g[j][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < RF; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const float f = xb[16 * t + 4 * fg + e][16 * h + fr];
#pragma unroll
            for (int j = 0; j < CF; ++j) g[j][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(f, pf[j][t][e], g[j][h], 0, 0, 0);
          }
#pragma unroll
      for (int j = 0; j < CF; ++j) {
#pragma unroll
        for (int h = 0; h < 4; ++h) *(f32x4*)&out[wid][fr][16 * h + 4 * fg] = g[j][h];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = c0 + 16 * j + 4 * q + fg, k = step * KC + 4 * fr;
          const f32x4 f = *(const f32x4*)&out[wid][4 * q + fg][4 * fr];
          const float v[4] = {f[0] * scale, f[1] * scale, f[2] * scale, f[3] * scale};
          if (c < p.n) store_some(p.dW + (int64_t)c * p.d + k, p.d - k, v);
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
}

// A share of dx = P W: 64 columns (blockIdx.x of them) of the classes from blockIdx.y `per` on, 16 a step of a wave.  A lane reads 16
// bytes of a class, four columns of the matrix instructions', and the classes' P.
template <int RF>
__global__ __launch_bounds__(256) void k_loss_few_dx(const int32_t* n_have, const float* P, const float* W, int n, int d, int per,
                                                     int64_t rows, float* part) {
  __shared__ __align__(16) float sums[2][16 * RF][LDC];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, fr = lane & 15, fg = lane >> 4;
  const int k = (int)blockIdx.x * KC + 4 * fr, count = *n_have;
  if (count == 0) return;
  const int64_t first = (int64_t)blockIdx.y * per, end = min(first + per, (int64_t)n);
  float wv[4][4], pv[4][RF];
  const auto load = [&](int64_t c) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t at = c + 4 * t + fg, use = min(at, (int64_t)n - 1);
      load_some(W + use * d + k, d - k, wv[t]);
#pragma unroll
      for (int i = 0; i < RF; ++i) {
        pv[t][i] = P[use * (16 * RF) + 16 * i + fr];
        if (at >= end) pv[t][i] = 0.f;
      }
      if (at >= end) wv[t][0] = wv[t][1] = wv[t][2] = wv[t][3] = 0.f;
    }
  };
  f32x4 acc[RF][4];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  int64_t c = first + 16 * wid;
  if (c < end) load(c);
  for (; c < end; c += 64) {
    float w[4][4], q[4][RF];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[t][e] = wv[t][e];
#pragma unroll
      for (int i = 0; i < RF; ++i) q[t][i] = pv[t][i];
    }
    if (c + 64 < end) load(c + 64);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < RF; ++i) acc[i][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[t][i], w[t][e], acc[i][e], 0, 0, 0);
  }
  // (a lane has columns k .. k + 3 of the rows 16 i + 4 fg + q; the waves' sums are added by halves)
#pragma unroll
  for (int half = 2; half > 0; half >>= 1) {
    if (wid >= half && wid < 2 * half) {
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(f32x4*)&sums[wid - half][16 * i + 4 * fg + q][4 * fr] = f32x4{acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]};
    }
    __syncthreads();
    if (wid < half) {
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 o = *(const f32x4*)&sums[wid][16 * i + 4 * fg + q][4 * fr];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][e][q] += o[e];
        }
    }
    __syncthreads();
  }
  if (wid) return;
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = 16 * i + 4 * fg + q;
      const float v[4] = {acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]};
      if (r < count) store_some(part + ((int64_t)blockIdx.y * rows + r) * d + k, d - k, v);
    }
}

// The sums of the blocks that shared a product's: rows of dx (idx given: the rows with a label) or of dW.  `by` threads of a
// block add up every by-th share of the same four elements.
__global__ __launch_bounds__(256) void k_loss_shares(const int32_t* count, const int32_t* idx, const float* part, int split, int by,
                                                     int64_t rows, int d, const float* dloss, int add, float* out, int64_t ldo) {
  __shared__ float4 sums[256];
  const uint32_t dv = (uint32_t)cdiv(d, 4), each = 256 / by, at = threadIdx.x % each, k = threadIdx.x / each;
  const uint32_t e = blockIdx.x * each + at;
  const int64_t r = e / dv, n = *count;
  const int c = (int)(e % dv) * 4;
  const bool mine = r < (idx ? n : rows);
  float v[4] = {0.f, 0.f, 0.f, 0.f}, w[4];
  for (int s = (int)k; mine && s < split; s += by) {
    load_some(part + (s * rows + r) * d + c, d - c, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += w[i];
  }
  if (by > 1) {
    sums[threadIdx.x] = make_float4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    for (int j = 1; k == 0 && j < by; ++j) {
      const float4 o = sums[j * each + at];
      v[0] += o.x, v[1] += o.y, v[2] += o.z, v[3] += o.w;
    }
  }
  if (!mine || k) return;
  float* o = out + (idx ? (int64_t)idx[r] : r) * ldo + c;
  const float scale = loss_scale(n, dloss);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] *= scale;
  if (add) {
    load_some(o, d - c, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += w[i];
  }
  store_some(o, d - c, v);
}

// --------------------------------------------------------------------------- rows' sums

// R rows a block, THREADS / R threads to each: joins the tiles' (largest, sum) and leaves the row's, its loss, and the block's sum;
// of one block the mean too.  (A mean by the last of many blocks to be done in the same launch needs a fence of each, which took
// longer than the launch: 18 us for 9 + 5, 7,373 rows.)
template <int R, int THREADS>
__global__ __launch_bounds__(THREADS) void k_loss_join(const int32_t* count, const int32_t* idx, const float2* part, int tiles,
                                                       int64_t ld_part, const float* at_label, float2* stat, float* row_loss,
                                                       double* sums, float* loss) {
  constexpr int EACH = THREADS / R;
  __shared__ float2 s[EACH][R + 1];
  __shared__ double l[R];
  const int j = threadIdx.x % R, k = threadIdx.x / R;
  const int64_t n = *count, r = (int64_t)blockIdx.x * R + j;
  if ((int64_t)blockIdx.x * R >= n) {
    if (gridDim.x == 1 && threadIdx.x == 0) *loss = 0.f;
    return;
  }
  float2 q = make_float2(-INFINITY, 0.f);
  const auto add = [&](float2 o) {
    const float m = fmaxf(q.x, o.x), from = base_of(m);
    q.y = q.y * expf(q.x - from) + o.y * expf(o.x - from);
    q.x = m;
  };
  if (r < n)
    for (int t = k; t < tiles; t += 8 * EACH) {   // (those past the last one: nothing)
      float2 o[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) o[u] = t + EACH * u < tiles ? part[(t + EACH * u) * ld_part + r] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int u = 0; u < 8; ++u) add(o[u]);
    }
  s[k][j] = q;
  for (int h = EACH / 2; h > 0; h >>= 1) {
    __syncthreads();
    if (k < h) {
      add(s[k + h][j]);
      s[k][j] = q;
    }
  }
  if (k == 0) {
    double v = 0.0;
    if (r < n) {
      const float f = (q.x - at_label[r]) + logf(q.y);
      stat[r] = make_float2(q.x, 1.f / q.y);
      if (row_loss) row_loss[idx[r]] = f;
      v = f;
    }
    l[j] = v;
  }
  __syncthreads();
  if (threadIdx.x) return;
  double v = 0.0;
  for (int i = 0; i < R; ++i) v += l[i];
  if (gridDim.x == 1) *loss = (float)(v / (double)n);
  else sums[blockIdx.x] = v;
}

constexpr int JOIN = 16;   // rows of a block of k_loss_join where there are several
__global__ __launch_bounds__(256) void k_loss_mean(const int32_t* count, const double* sums, float* loss) {
  __shared__ double s[256];
  const int64_t n = *count, blocks = cdiv(n, JOIN);
  double v = 0.0;
  for (int64_t i = threadIdx.x; i < blocks; i += 256) v += sums[i];
  s[threadIdx.x] = v;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) s[threadIdx.x] += s[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *loss = n > 0 ? (float)(s[0] / (double)n) : 0.f;
}

// db of a piece, from the column sums of each `per` rows.
__global__ __launch_bounds__(256) void k_loss_db(const int32_t* count, const float* part, int64_t ld, int64_t per, int64_t cols,
                                                 const float* dloss, float* db) {
  __shared__ float s[16][17];
  const int j = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int64_t c = (int64_t)blockIdx.x * 16 + j, n = *count, parts = cdiv(n, per);
  float v = 0.f;
  if (c < cols)
    for (int64_t i = k; i < parts; i += 16) v += part[i * ld + c];
  s[k][j] = v;
  __syncthreads();
  if (k || c >= cols) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += s[i][j];
  db[c] = v * loss_scale(n, dloss);
}

// --------------------------------------------------------------------------- memory

size_t al(size_t b) { return (b + 255) & ~size_t(255); }

// Bytes of P in memory at a time (where a piece is more than 256 classes wide).  With 2^28, 2^30 and 2^31, gradients of 8,192 x 32,768 x
// 1,024 in bfloat16 4,586, 4,033 and 4,006 us.
constexpr size_t PIECE = size_t(1) << 30;

// Elements from a row to the next one in memory of our own: whole 128 bytes, an odd number of them, so that a column of rows is
// not in a few of the memory's channels.
int64_t stride(int64_t width) { return up(width, PAD) | PAD; }

struct Plan {
  bool bf, copy;             // bfloat16 operands; their W is copied (its rows are not whole 16 bytes at 16-byte addresses)
  bool few, few_back;        // float32 operands of so few rows that the forward, and the backward too, read W as it is
  int dp;                    // padded width
  int64_t Rp, width;         // padded rows; classes of a piece
};
// Rows of float32 that k_loss_few's forward takes: up to 192, or 256 where its blocks are all on the card at once (three a CU).  The
// forward in parts and by it, us: 92 x 48,988 x 1,024 215 and 137, 129 x 38,544 x 1,024 222 and 174, 192 x 60,000 x 200 79 and 83,
// 192 x 150,000 x 512 403 and 319; 200 x 9,000 x 100 26 and 20, 250 x 3,000 x 1,024 81 and 38; 256 x 20,000 x 768 (1,252 blocks) 94
// and 101, 256 x 60,000 x 200 81 and 107, 256 x 150,000 x 1,024 824 and 766.  The backward by it takes up to 64: 64 x 30,000 x
// 512 with the forward 218 and 130; 92 x 48,988 x 1,024 alone 414, and in groups of 64 rows 507.
bool few_rows(const mtgnn_loss_dims* d, int64_t rows) {
  return rows <= 192 || (rows <= FEW && cdiv(d->n, 64) * cdiv(rows, 64) <= 768);
}
Plan plan(const mtgnn_loss_dims* d, int64_t rows, const void* W) {
  Plan p;
  p.bf = d->dtype == MTGNN_BF16;
  p.dp = (int)stride(d->d);
  p.copy = p.bf && (d->d % 8 != 0 || (uintptr_t)W % 16 != 0);
  p.few = !p.bf && few_rows(d, rows);
  p.few_back = p.few && rows <= 64;
  p.Rp = up(rows, PAD);
  // (rows of P are up to 64 elements longer than a piece is wide)
  const int64_t most = std::max<int64_t>(256, ((int64_t)(PIECE / (6 * (size_t)p.Rp)) - PAD) / 256 * 256), pieces = cdiv(d->n, most);
  p.width = pieces == 1 ? up(d->n, PAD) : up(cdiv(d->n, pieces), 256);
  return p;
}

struct Kept {                // what the forward leaves for the backward
  int32_t* count;
  int32_t *idx, *lab;
  float2* stat;
  uint16_t* xc;              // x's rows: as they are, or float32 in three parts
};
size_t kept_bytes(const Plan& p) { return 256 + 2 * al(4 * p.Rp) + al(8 * p.Rp) + al(2 * (size_t)(p.bf ? 1 : p.few ? 2 : 3) * p.Rp * p.dp); }
Kept kept(void* at, const Plan& p) {
  Kept k;
  char* w = (char*)at;
  k.count = (int32_t*)w;
  k.idx = (int32_t*)(w += 256);
  k.lab = (int32_t*)(w += al(4 * p.Rp));
  k.stat = (float2*)(w += al(4 * p.Rp));
  k.xc = (uint16_t*)(w += al(8 * p.Rp));
  return k;
}

// A product's tiles, and the blocks that share a tile's sum.
struct Tiling {
  int tr, tc, split;
  int64_t tiles(int64_t rows, int64_t cols) const { return cdiv(rows, tr) * cdiv(cols, tc); }
};
// Of the logits: wide tiles for few rows (33 x 100,003 x 520 is reading W: 24 us, 4.3 TB/s; the whole forward in wide, small and large
// tiles 38, 47 and 58 us, 64 x 30,000 x 1,024 33, 32 and 41, 40 x 9,000 x 100 19, 19 and 21); else large ones unless the last
// round of them leaves too much of the card empty: the forward in large and small ones, us, 3,000 x 6,000 x 512 in float32 (288
// large tiles) 160 and 136, 2,000 x 30,000 x 512 (944) 332 and 374, 4,000 x 9,001 x 512 in bfloat16 (576) 75 and 72, 4,000 x
// 16,000 x 512 (1,008) 100 and 107.
Tiling tiling(int64_t rows, int64_t cols) {
  if (rows <= 64) return Tiling{64, 256, 1};
  const Tiling big{256, 256, 1}, small{128, 128, 1};
  return cdiv(big.tiles(rows, cols), 256) * 100 <= cdiv(small.tiles(rows, cols), 512) * 56 ? big : small;
}
// Of a gradient, with sums of `steps` steps: the tiles and shares that are done first, in us: rounds of blocks, a step of 1.53 in large
// tiles and 1 in small ones, two of which a compute unit has, 6 steps a block beside its own, and the shares' way to memory and
// back, with a launch.  (Gradients and logits, us, in small tiles alone, large ones alone and as chosen here: 4,000 x 9,001 x 100
// in float32 344, 386, 342; 500 x 20,000 x 512 345, 350, 341; 3,000 x 6,000 x 512 523, 485, 488; 8,192 x 32,768 x 1,024 in
// bfloat16 4,639, 3,985, 3,980; 1,000 x 30,000 x 1,024 574, 526, 519.)
Tiling tiling(int64_t rows, int64_t cols, int64_t steps) {
  Tiling best{256, 256, 1};
  double least = INFINITY;
  const double size = (double)rows * (double)cols / 8e5;
  for (const Tiling g : {Tiling{256, 256, 1}, Tiling{128, 128, 1}}) {
    const int64_t t = g.tiles(rows, cols), slots = g.tr == 256 ? 256 : 512;
    const double step = g.tr == 256 ? 1.53 : 1.;
    const auto look = [&](int64_t s) {
      s = std::max<int64_t>(1, std::min(s, steps / 8));
      const double cost = step * (double)(cdiv(t * s, slots) * (cdiv(steps, s) + 6)) + (s > 1 ? 1.4 * (6. + (double)s * size) : 0.);
      if (cost < least) least = cost, best = g, best.split = (int)s;
    };
    look(1);
    for (int k = 1; k <= 4; ++k) look(k * slots / t);   // whole rounds,
    // or so many that more would gain less than they cost
    if (t < slots) look(std::min(slots / t, (int64_t)std::sqrt((double)steps / size)));
  }
  return best;
}
int row_frags(int64_t rows) { return rows > 32 ? 4 : rows > 16 ? 2 : 1; }
// Classes of a share of k_loss_few_dx: enough blocks to fill the card, each of a few steps at least.
int few_per(const mtgnn_loss_dims* d) {
  const int64_t chunks = cdiv(d->d, KC), shares = std::max<int64_t>(1, std::min<int64_t>(cdiv(2048, chunks), d->n / 256));
  return (int)up(cdiv(d->n, shares), 64);
}
// Classes of a block of the forward's k_loss_few: more for short rows of many classes, whose tiles then take less time to join
// (128 and 64, the whole forward: 16 x 190,000 x 200 42 and 47 us, 14 x 142,281 x 1,024 145 and 129, 64 x 9,000 x 1,024 53 and 38).
int few_classes(const mtgnn_loss_dims* d) { return d->n >= 32768 && d->d < 512 ? 128 : 64; }
// A forward's tiles of classes.
int64_t class_tiles(const mtgnn_loss_dims* d, const Plan& p, int64_t rows) {
  return cdiv(d->n, p.few ? few_classes(d) : tiling(rows, d->n).tc);
}
struct Shares {
  Tiling dx, dw;             // of a piece
  size_t bytes;
};
Shares shares_of(const mtgnn_loss_dims* d, const Plan& p, int64_t rows, int64_t cols) {
  const int segs = p.bf ? 3 : 6;
  Shares s;
  s.dx = tiling(rows, d->d, segs * cdiv(cols, KS));
  s.dw = tiling(cols, d->d, segs * cdiv(rows, KS));
  s.bytes = std::max(s.dx.split > 1 ? 4 * (size_t)s.dx.split * rows * d->d : 0,
                     s.dw.split > 1 ? 4 * (size_t)s.dw.split * cols * d->d : 0);
  return s;
}

template <int KIND>
mtgnn_status product(Prod p, const Tiling& t, hipStream_t s) {
  p.tr = cdiv(p.rows, t.tr);
  p.tc = cdiv(p.cols, t.tc);
  p.split = t.split;
  const unsigned grid = (unsigned)(p.tr * p.tc * p.split);
  {
    TimedScope ts(site::Generic::name, s),
        kind(KIND == STAT ? "loss_stat" : KIND == PROB ? "loss_prob" : KIND == DX ? "loss_dx" : "loss_dw", s);
    if (t.tr == 256) k_loss_product<KIND, 256, 256><<<grid, 512, 0, s>>>(p);
    else if (t.tr == 128) k_loss_product<KIND, 128, 128><<<grid, 256, 0, s>>>(p);
    else if constexpr (KIND == STAT || KIND == PROB) k_loss_product<KIND, 64, 256><<<grid, 256, 0, s>>>(p);
  }
  MTGNN_CHECK_LAUNCH("loss_product");
  return MTGNN_OK;
}
mtgnn_status join_shares(const Prod& p, int split, const float* part, hipStream_t s) {
  const int by = split > 32 ? 16 : split > 8 ? 4 : 1;   // (many shares are of few elements)
  k_loss_shares<<<(unsigned)cdiv(p.rows * cdiv(p.cols, 4), 256 / by), 256, 0, s>>>(p.count, p.idx, part, split, by, p.rows, (int)p.cols,
                                                                                   p.dloss, p.add, p.out, p.ldo);
  MTGNN_CHECK_LAUNCH("loss_shares");
  return MTGNN_OK;
}
// A gradient's product, shared by `split` blocks a tile through `part`.
template <int KIND>
mtgnn_status gradient(const Prod& p, const Tiling& t, float* part, hipStream_t s) {
  if (t.split <= 1) return product<KIND>(p, t, s);
  Prod q = p;
  q.out = part;
  q.ldo = p.cols;
  MTGNN_TRY(product<KIND>(q, t, s));
  return join_shares(p, t.split, part, s);
}
mtgnn_status few(const Few& p, int tc, hipStream_t s) {
  const int rf = row_frags(p.max_rows);
  const unsigned grid = (unsigned)(cdiv(p.n, tc) * p.groups);
  {
    TimedScope ts(site::Generic::name, s), kind("loss_stat", s);
    if (tc == 128) {
      if (rf == 4) k_loss_few<4, 2, false><<<grid, 256, 0, s>>>(p);
      else if (rf == 2) k_loss_few<2, 2, false><<<grid, 256, 0, s>>>(p);
      else k_loss_few<1, 2, false><<<grid, 256, 0, s>>>(p);
    } else if (rf == 4) k_loss_few<4, 1, false><<<grid, 256, 0, s>>>(p);
    else if (rf == 2) k_loss_few<2, 1, false><<<grid, 256, 0, s>>>(p);
    else k_loss_few<1, 1, false><<<grid, 256, 0, s>>>(p);
  }
  MTGNN_CHECK_LAUNCH("loss_few");
  return MTGNN_OK;
}
mtgnn_status few_back(const Few& p, hipStream_t s) {
  const int rf = row_frags(p.max_rows);
  const unsigned grid = (unsigned)cdiv(p.n, 64);
  {
    TimedScope ts(site::Generic::name, s), kind("loss_prob", s);
    if (rf == 4) k_loss_few<4, 1, true><<<grid, 256, 0, s>>>(p);
    else if (rf == 2) k_loss_few<2, 1, true><<<grid, 256, 0, s>>>(p);
    else k_loss_few<1, 1, true><<<grid, 256, 0, s>>>(p);
  }
  MTGNN_CHECK_LAUNCH("loss_few_back");
  return MTGNN_OK;
}

// The products of parts, the smaller ones first: of float32 operands (A in three parts, B too: both) six, of P and a bfloat16 one three.
void segments(Prod& p, bool a, bool b) {
  constexpr auto code = [](int q0, int q1, int q2, int q3, int q4, int q5) {
    return (uint32_t)(q0 | q1 << 2 | q2 << 4 | q3 << 6 | q4 << 8 | q5 << 10);
  };
  p.segs = b ? 6 : a ? 3 : 1;
  p.codeA = b ? code(2, 0, 1, 1, 0, 0) : a ? code(2, 1, 0, 0, 0, 0) : 0u;
  p.codeB = b ? code(0, 2, 1, 0, 1, 0) : 0u;
}

unsigned table_blocks(int64_t n, int dp) { return (unsigned)cdiv(up(n, PAD) * (dp / 8), 256); }

}  // namespace

bool loss_fits(const mtgnn_loss_dims* d, int64_t rows) {
  constexpr int64_t MAX = (int64_t(1) << 32) - (int64_t(1) << 20);
  const auto tiles = [](int64_t r, int64_t c) { return cdiv(r, 128) * cdiv(c, 128) * 256; };   // (shares only of few)
  const int64_t units = stride(d->d) / 8, W = (d->n + PAD) * units, x = (rows + PAD) * units;   // threads that lay out a matrix
  return tiles(rows, d->n) < MAX && tiles(rows, d->d) < MAX && tiles(d->n, d->d) < MAX && W + x + rows * cdiv(d->d, 4) < MAX &&
         W + rows * 16 < MAX && std::max<int64_t>(rows, d->n) * cdiv(d->d, 4) < MAX;
}

size_t loss_save(const mtgnn_loss_dims* d, int64_t rows) { return kept_bytes(plan(d, rows, nullptr)); }

size_t loss_ws(const mtgnn_loss_dims* d, int64_t rows, bool back) {
  const Plan p = plan(d, rows, nullptr);   // (W's address is not known yet: there is room for its copy whatever it is)
  const size_t t = al(2 * (size_t)up(d->n, PAD) * p.dp);   // a part of W
  if (!back)
    return kept_bytes(p) + (p.bf ? t : p.few ? 0 : 3 * t) + al(4 * cdiv(p.Rp, CHUNK)) +
           al(8 * (size_t)class_tiles(d, p, rows) * p.Rp) + al(4 * p.Rp) + al(8 * cdiv(p.Rp, JOIN));
  if (p.few_back) return al(4 * (size_t)d->n * 16 * row_frags(rows)) + al(4 * (size_t)cdiv(d->n, few_per(d)) * rows * d->d);
  const int64_t last = d->n % p.width ? d->n % p.width : std::min<int64_t>(d->n, p.width);
  const size_t part = std::max(shares_of(d, p, rows, std::min<int64_t>(d->n, p.width)).bytes, shares_of(d, p, rows, last).bytes);
  return (p.bf ? t : 3 * t + (p.few ? al(6 * (size_t)p.Rp * p.dp) : 0)) + al(6 * (size_t)p.Rp * stride(p.width)) +
         al(4 * (size_t)cdiv(p.Rp, 64) * stride(p.width)) + al(part);
}

mtgnn_status loss_impl(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const void* W, const float* b,
                       const int32_t* label, const mtgnn_loss_dims* d, float* loss, float* row_loss, void* save, void* ws,
                       hipStream_t s) {
  const Plan p = plan(d, max_rows, W);
  const Kept k = kept(save ? save : ws, p);
  const Tiling tl = tiling(max_rows, d->n);
  char* w = (char*)ws + kept_bytes(p);
  const auto take = [&](size_t bytes) {
    char* at = w;
    w += al(bytes);
    return at;
  };
  const size_t plane = (size_t)up(d->n, PAD) * p.dp;
  uint16_t* tbl = (uint16_t*)take(p.bf ? (p.copy ? 2 * plane : 0) : p.few ? 0 : 6 * plane);
  int32_t* counts = (int32_t*)take(4 * cdiv(p.Rp, CHUNK));
  const int tiles = (int)class_tiles(d, p, max_rows);
  float2* part = (float2*)take(8 * (size_t)tiles * p.Rp);
  float* at_label = (float*)take(4 * p.Rp);
  double* sums = (double*)take(8 * cdiv(p.Rp, JOIN));
  const unsigned blocks = (unsigned)(cdiv(max_rows, ROWS) + PAD / ROWS), tb = p.bf && !p.copy ? 0 : table_blocks(d->n, p.dp);
  const auto lay = [&](auto* xt, auto* Wt) -> mtgnn_status {
    const bool alone = max_rows <= CHUNK;
    if (!alone) k_loss_count<<<(unsigned)cdiv(max_rows, CHUNK), 256, 0, s>>>(label, n_rows, max_rows, d->n, counts);
    MTGNN_CHECK_LAUNCH("loss_count");
    k_loss_lay<<<blocks + tb, 256, 0, s>>>(xt, ldx, label, n_rows, max_rows, d->n, d->d, p.dp, alone ? nullptr : counts, k.count,
                                           k.idx, k.lab, k.xc, p.Rp * p.dp, row_loss, blocks, Wt, tbl);
    MTGNN_CHECK_LAUNCH("loss_lay");
    return MTGNN_OK;
  };
  if (!p.few) MTGNN_TRY(p.bf ? lay((const uint16_t*)x, (const uint16_t*)W) : lay((const float*)x, (const float*)W));
  Prod q{};
  q.A = k.xc; q.lda = p.dp; q.planeA = p.Rp * p.dp;
  q.B = tbl; q.ldb = q.endB = p.dp; q.planeB = plane;
  if (p.bf && !p.copy) q.B = (const uint16_t*)W, q.ldb = q.endB = d->d;
  segments(q, !p.bf, !p.bf);
  q.rows = max_rows; q.cols = d->n; q.K = up(d->d, KS); q.count = k.count;
  q.b = b; q.lab = k.lab; q.part = part; q.ld_part = p.Rp; q.at_label = at_label;
  if (p.few) {
    Few f{};
    f.x = (const float*)x; f.ldx = ldx; f.W = (const float*)W; f.b = b;
    f.label = label; f.n_rows = n_rows; f.max_rows = max_rows; f.n = d->n; f.d = d->d;
    f.count = k.count; f.idx = k.idx; f.lab = k.lab; f.xc = save ? (float*)k.xc : nullptr; f.dp = p.dp;
    f.part = part; f.ld_part = p.Rp; f.at_label = at_label; f.row_loss = row_loss;
    f.groups = (int)cdiv(max_rows, 64);
    MTGNN_TRY(few(f, few_classes(d), s));
  } else {
    MTGNN_TRY(product<STAT>(q, tl, s));
  }
  // The whole forward, us: with 64 threads to a row, not 16, where there are more tiles than those request at once, 33 x 100,003 x 520
  // (391 tiles) 42 -> 38; with one block, and no launch for the mean, 17 x 9,000 x 100 (141 tiles) 18.4 -> 15.5, but
  // 14 x 142,281 x 1,024 (2,224 tiles) 130 -> 157.
  const auto join = [&](auto kernel, int rows, int threads) -> mtgnn_status {
    kernel<<<(unsigned)cdiv(max_rows, rows), threads, 0, s>>>(k.count, k.idx, part, tiles, p.Rp, at_label, k.stat, row_loss, sums,
                                                              loss);
    MTGNN_CHECK_LAUNCH("loss_join");
    return MTGNN_OK;
  };
  if (max_rows <= 64 && tiles <= 256) return join(k_loss_join<64, 1024>, 64, 1024);
  MTGNN_TRY(tiles > 128 ? join(k_loss_join<JOIN, 1024>, JOIN, 1024) : join(k_loss_join<JOIN, 256>, JOIN, 256));
  if (max_rows <= JOIN) return MTGNN_OK;
  k_loss_mean<<<1, 256, 0, s>>>(k.count, sums, loss);
  MTGNN_CHECK_LAUNCH("loss_mean");
  return MTGNN_OK;
}

mtgnn_status loss_bwd_impl(const int32_t* n_rows, int64_t max_rows, const void* W, const float* b, const int32_t* label,
                           const mtgnn_loss_dims* d, const void* save, const float* dloss, float* dx, int64_t lddx, float* dW,
                           float* db, void* ws, hipStream_t s) {
  const Plan p = plan(d, max_rows, W);
  const Kept k = kept((void*)save, p);
  char* w = (char*)ws;
  const auto take = [&](size_t bytes) {
    char* at = w;
    w += al(bytes);
    return at;
  };
  if (p.few_back) {
    const int rf = row_frags(max_rows), per = few_per(d);
    float* P = (float*)take(4 * (size_t)d->n * 16 * rf);
    Few f{};
    f.W = (const float*)W; f.b = b; f.max_rows = max_rows; f.n = d->n; f.d = d->d;
    f.count = k.count; f.idx = k.idx; f.lab = k.lab; f.xc = (float*)k.xc; f.dp = p.dp;
    f.stat = k.stat; f.dloss = dloss; f.P = dx ? P : nullptr; f.db = db; f.dW = dW;
    f.groups = 1;
    MTGNN_TRY(few_back(f, s));
    if (!dx) return MTGNN_OK;
    const unsigned zb = (unsigned)cdiv(max_rows * cdiv(d->d, 4), 256);
    k_loss_back_lay<float><<<zb, 256, 0, s>>>(label, n_rows, max_rows, d->n, d->d, dx, lddx, zb, nullptr, 0, 0, nullptr, 0, nullptr, 0,
                                              0, nullptr);
    MTGNN_CHECK_LAUNCH("loss_back_lay");
    Prod r{};
    r.rows = max_rows; r.cols = d->d; r.count = k.count; r.idx = k.idx; r.dloss = dloss; r.out = dx; r.ldo = lddx;
    const dim3 grid((unsigned)cdiv(d->d, KC), (unsigned)cdiv(d->n, per));
    {
      TimedScope ts(site::Generic::name, s), kind("loss_dx", s);
      if (rf == 4) k_loss_few_dx<4><<<grid, 256, 0, s>>>(k.count, P, (const float*)W, d->n, d->d, per, max_rows, (float*)w);
      else if (rf == 2) k_loss_few_dx<2><<<grid, 256, 0, s>>>(k.count, P, (const float*)W, d->n, d->d, per, max_rows, (float*)w);
      else k_loss_few_dx<1><<<grid, 256, 0, s>>>(k.count, P, (const float*)W, d->n, d->d, per, max_rows, (float*)w);
    }
    MTGNN_CHECK_LAUNCH("loss_few_dx");
    return join_shares(r, (int)grid.y, (float*)w, s);
  }
  const bool in_place = p.bf && !p.copy;
  const int64_t plane = up(d->n, PAD) * p.dp, planeX = p.Rp * p.dp;
  // W, or what is behind the last whole step of one in place: its rows from w0 on
  const int64_t w0 = in_place ? d->n / KS * KS : 0;
  const int wdp = in_place ? d->d : p.dp;
  uint16_t* tbl = (uint16_t*)take(2 * (size_t)(p.bf ? 1 : 3) * up(d->n - w0, PAD) * wdp);
  uint16_t* xh = p.few ? (uint16_t*)take(6 * (size_t)planeX) : k.xc;
  uint16_t* P = (uint16_t*)take(6 * (size_t)p.Rp * stride(p.width));
  float* cols_part = (float*)take(4 * (size_t)cdiv(p.Rp, 64) * stride(p.width));
  float* part = (float*)w;
  const unsigned zb = dx ? (unsigned)cdiv(max_rows * cdiv(d->d, 4), 256) : 0, tb = table_blocks(d->n - w0, wdp);
  const auto lay = [&](auto* Wt) -> mtgnn_status {
    const unsigned grid = zb + tb + (p.few ? table_blocks(p.Rp, p.dp) : 0);
    if (grid > 0)
      k_loss_back_lay<<<grid, 256, 0, s>>>(label, n_rows, max_rows, d->n, d->d, dx, lddx, zb, Wt + w0 * d->d, d->n - w0, wdp, tbl, tb,
                                           (decltype(Wt))k.xc, p.Rp, p.dp, xh);
    MTGNN_CHECK_LAUNCH("loss_back_lay");
    return MTGNN_OK;
  };
  MTGNN_TRY(p.bf ? lay((const uint16_t*)W) : lay((const float*)W));
  // W from class c on: what the forward's product has, so its logits are formed again (those of k_loss_few differ by their rounding)
  const auto table = [&](Prod& q, int64_t c) {
    q.B = in_place ? (const uint16_t*)W + c * d->d : tbl + c * p.dp;
    q.ldb = wdp;
    q.planeB = plane;
  };
  for (int64_t c = 0; c < d->n; c += p.width) {
    const int64_t cols = std::min<int64_t>(p.width, d->n - c), ldp = stride(cols);
    const Shares sh = shares_of(d, p, max_rows, cols);
    const Tiling tl = tiling(max_rows, cols);
    Prod q{};
    q.A = xh; q.lda = p.dp; q.planeA = planeX;
    table(q, c);
    q.endB = q.ldb;
    q.rows = max_rows; q.cols = cols; q.K = up(d->d, KS); q.count = k.count;
    q.b = b ? b + c : nullptr; q.lab = k.lab; q.c0 = c; q.stat = k.stat;
    q.P = P; q.ldp = ldp; q.planeP = p.Rp * ldp;
    q.cols_part = db ? cols_part : nullptr;
    segments(q, !p.bf, !p.bf);
    MTGNN_TRY(product<PROB>(q, tl, s));
    if (db) {
      k_loss_db<<<(unsigned)cdiv(cols, 16), 256, 0, s>>>(k.count, cols_part, ldp, tl.tr == 64 ? 64 : tl.tr / 2, cols, dloss, db + c);
      MTGNN_CHECK_LAUNCH("loss_db");
    }
    Prod g{};
    g.A = P; g.lda = g.dimA = ldp; g.planeA = p.Rp * ldp;
    g.cols = d->d; g.count = k.count; g.dloss = dloss;
    segments(g, true, !p.bf);
    if (dx) {
      Prod r = g;
      table(r, c);
      r.dimB = r.ldb; r.endB = up(d->n, in_place ? 1 : PAD) - c; r.tail = tbl - r.B;
      r.rows = max_rows; r.K = cols; r.idx = k.idx; r.out = dx; r.ldo = lddx; r.add = c > 0;
      MTGNN_TRY((gradient<DX>(r, sh.dx, part, s)));
    }
    if (dW) {
      Prod r = g;
      r.B = xh; r.ldb = r.dimB = p.dp; r.planeB = planeX;
      r.rows = cols; r.out = dW + c * d->d; r.ldo = d->d;
      MTGNN_TRY((gradient<DW>(r, sh.dw, part, s)));
    }
  }
  return MTGNN_OK;
}

}  // namespace mtgnn
