// Linear layer with bias, activation and residual, and its backward:
//   y = act(x W^T + b) + residual;   g = dy act'(pre),  dx = g W,  dW = g^T x,  db = sum of g.
//
// All three products run in one kernel, out[r][c] = sum_k R(r, k) C(c, k), on the bfloat16 matrix instructions.  A
// bfloat16 operand enters as it is; a float32 one as three bfloat16 parts (24 bits, bf16_split.h), split as its tile is
// staged: three products for one such operand, six for two (the three smallest, below 2^-26 of the
// whole, are left out), which is still 2.6 times the rate of the float32 matrix instructions.  Results are
// exact to float32 either way.
//
// A block of four waves makes a T x T tile (T = 128 or 64), each wave a quarter of it.  Operands pass through
// registers into LDS in 16-byte units of eight k, from rows that are contiguous along k or across it; the next
// step's loads are in flight while the matrix instructions work on this one.  A unit's place in its row is
// swizzled by the row, so that eight lanes' reads and writes of 16 bytes meet every bank once.  The matrix instruction's
// first operand is C: a lane then holds four neighbouring columns of a row.  Tiles leave through LDS, so that
// rows are written in 128 to 256 bytes, and the epilogue is a loop and not 64 copies of it.
//
// Measured (us, kernel trace, median of 53; calls in a row hide 1 or 2 of each): data gradient 8,192 x 2,048 -> 1,024 from a
// float32 slope (three products) 134, 770 TFLOP/s of products; weight gradient 137 + 11 for the shares; there the LDS
// traffic of the three parts (reads and writes as long as the matrix instructions) bounds it.  Float32 8,000 x 300 -> 200:
// 19 (17 in a row), five dependent steps of 500 blocks, so latency.
#include <algorithm>

#include "bf16_split.h"
#include "gemm.h"
#include "ops.h"
#include "seq.h"

namespace mtgnn {

namespace {

constexpr int NT = 256;

struct ProdP {
  const void *R, *C;
  int64_t ldR, ldC;
  int64_t rows, cols, K;           // rows of R and C, length of the sums
  const int32_t *rows_dev, *K_dev; // device counts that bound them, or NULL
  int aligned;                     // every row of both operands starts at a multiple of 16 bytes
  int64_t tc, tiles;               // tiles of a row of tiles, tiles in all
  int split;                       // blocks that share a tile's sum
  // output: float32 sums (o, split x rows x cols of them where split > 1), or the layer's epilogue (y given)
  float* o;
  int64_t ldo;
  const float* b;
  const void* res;
  int64_t ldr;
  void* y;
  int64_t ldy;
  float* pre;
  int act;
};

// Sixteen bytes at any element's address (the loads take it; a row of an odd length is at no other).
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef words4 words4_at4 __attribute__((aligned(4)));
typedef words4 words4_at2 __attribute__((aligned(2)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef words2 words2_at4 __attribute__((aligned(4)));
typedef uint32_t word_at2 __attribute__((aligned(2)));

// One operand's share of a tile in a thread's registers: U units of eight k.  Where rows are contiguous across k, a thread's
// units are of two neighbouring rows, whose values at one k come by one load: weight gradient 145 us against 172 (8,192
// rows, 2,048 x 1,024, tiles of 128).  Not of float32 in tiles of 64, where half a wave's 256 bytes are a row's already: 51
// against 54 us with pairs (1,968 rows, 445 x 2,101).
template <bool F32, bool KC, int T, int KS>
struct Stage {
  static constexpr int U = T * KS / 8 / NT, CH = KS / 8, PL = F32 ? 3 : 1;
  static constexpr bool PAIR = !KC && (T == 128 || !F32);
  static_assert(U >= 1 && (!PAIR || U % 2 == 0), "a unit, or two rows of them, per thread");
  uint32_t v[U][F32 ? 8 : 4];
  __device__ __forceinline__ static int row(int u) {
    const int id = u * NT + threadIdx.x, pair = u / 2 * NT + threadIdx.x;
    return KC ? id / CH : PAIR ? pair % (T / 2) * 2 + u % 2 : id % T;
  }
  __device__ __forceinline__ static int chunk(int u) {
    const int id = u * NT + threadIdx.x, pair = u / 2 * NT + threadIdx.x;
    return KC ? id % CH : PAIR ? pair / (T / 2) : id / T;
  }
  using E = std::conditional_t<F32, uint32_t, uint16_t>;
  const E* q[U];   // of each unit: its row at k = 0
  int64_t ld;
  // rows r0 .. of the operand (the last one stands for those past it)
  __device__ __forceinline__ void at_rows(const void* p, int64_t ld_, int64_t rows, int64_t r0) {
    ld = ld_;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = min(r0 + row(u), rows - 1);
      q[u] = (const E*)p + (KC ? r * ld : r);
    }
  }
  // k0 .. k0 + KS - 1 (zeros from K on)
  __device__ __forceinline__ void load(int64_t k0, int64_t K) {
    if constexpr (KC) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + chunk(u) * 8;
        if (k + 8 > K) {
          load_each(u, k, K);
        } else if constexpr (F32) {
          const words4_at4* w = (const words4_at4*)(q[u] + k);
          const words4 a = w[0], b = w[1];
          v[u][0] = a.x; v[u][1] = a.y; v[u][2] = a.z; v[u][3] = a.w;
          v[u][4] = b.x; v[u][5] = b.y; v[u][6] = b.z; v[u][7] = b.w;
        } else {
          const words4 a = *(const words4_at2*)(q[u] + k);
          v[u][0] = a.x; v[u][1] = a.y; v[u][2] = a.z; v[u][3] = a.w;
        }
      }
    } else if constexpr (!PAIR) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + chunk(u) * 8;
        if (k0 + KS > K) {
          load_each(u, k, K);
          continue;
        }
        const E* w = q[u] + k * ld;
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = w[i * ld];
        put(u, e, 0, 8);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; u += 2) {
        const int64_t k = k0 + chunk(u) * 8;
        if (k0 + KS > K || q[u] == q[u + 1]) {   // (the last row is both where the row behind it does not exist)
          load_each(u, k, K);
          load_each(u + 1, k, K);
          continue;
        }
        const E* w = q[u] + k * ld;
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const words2 a = *(const words2_at4*)(w + i * ld);
            v[u][i] = a.x;
            v[u + 1][i] = a.y;
          }
        } else {
          uint32_t e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = *(const word_at2*)(w + i * ld);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[u][i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x05040100);
            v[u + 1][i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x07060302);
          }
        }
      }
    }
  }
  __device__ __forceinline__ void load_each(int u, int64_t k, int64_t K) {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t at = min(k + i, K - 1);
      e[i] = q[u][KC ? at : at * ld];
    }
    put(u, e, k, K);
  }
  __device__ __forceinline__ void put(int u, const uint32_t (&e)[8], int64_t k, int64_t K) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w = k + i < K ? e[i] : 0u;
      if constexpr (F32) v[u][i] = w;
      else if (i % 2 == 0) v[u][i / 2] = w;
      else v[u][i / 2] |= w << 16;
    }
  }
  // dst: [plane][T][KS] bfloat16, units swizzled
  __device__ __forceinline__ void store(uint32_t* dst) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t* d = dst + at(row(u), chunk(u));
      if constexpr (F32) {
        float x[8];
        uint32_t h[4], m[4], l[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[u][i]);
        split_words<false>(x, h, m, l);
        *(uint4*)d = make_uint4(h[0], h[1], h[2], h[3]);
        *(uint4*)(d + T * KS / 2) = make_uint4(m[0], m[1], m[2], m[3]);
        *(uint4*)(d + T * KS) = make_uint4(l[0], l[1], l[2], l[3]);
      } else {
        *(uint4*)d = make_uint4(v[u][0], v[u][1], v[u][2], v[u][3]);
      }
    }
  }
  // The swizzle: eight rows in turn meet every bank once, and eight even ones where units are stored by pairs of rows.
  __device__ __forceinline__ static int turn(int r) {
    const int t = CH == 4 ? r >> 1 & 3 : r & 7;
    return PAIR ? t ^ (r >> 3 & 1) : t;
  }
  // Word of unit c of row r in a plane.
  __device__ __forceinline__ static int at(int r, int c) {
    return r * (KS / 2) + (c ^ turn(r)) * 4;
  }
  __device__ __forceinline__ static bf16x8_t frag(const uint32_t* src, int plane, int r, int c) {
    return __builtin_bit_cast(bf16x8_t, *(const uint4*)(src + plane * (T * KS / 2) + at(r, c)));
  }
};

// Which tile and share of the sum this block makes.  Blocks run on the 8 XCDs in turn, each with its own L2: a
// contiguous eighth of the tiles to each, so the blocks of an XCD share rows of R.
__device__ __forceinline__ void my_tile(const ProdP& p, int64_t& tr, int64_t& tcol, int& share) {
  const int64_t L = blockIdx.x, n = p.tiles * p.split, full = n & ~int64_t(7);
  const int64_t V = L < full ? (L & 7) * (full >> 3) + (L >> 3) : L;
  share = (int)(V % p.split);
  const int64_t t = V / p.split;
  tr = t / p.tc;
  tcol = t % p.tc;
}

// One output by float32 products: what a sum that is not finite is made by again (a part of an infinite operand, or of
// one past the largest bfloat16, is infinite or NaN and meets the others' zeros).
template <bool RF, bool CF, bool RK, bool CK>
__device__ __attribute__((noinline)) float plain_sum(const void* R, int64_t ldR, const void* C, int64_t ldC, int64_t r,
                                                     int64_t c, int64_t k0, int64_t k1) {
  float v = 0.f;
  for (int64_t k = k0; k < k1 && v == v; k += 16) {   // a NaN stays one: the rest need not be read
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const int64_t at = min(k + u, k1 - 1);
      const int64_t a = RK ? r * ldR + at : at * ldR + r, b = CK ? c * ldC + at : at * ldC + c;
      const float x = RF ? ((const float*)R)[a] : bf16_to_f32(((const uint16_t*)R)[a]);
      const float w = CF ? ((const float*)C)[b] : bf16_to_f32(((const uint16_t*)C)[b]);
      v = k + u < k1 ? fmaf(x, w, v) : v;
    }
  }
  return v;
}

// Four columns (n of them) of a row: bias, activation, residual.  wide: y's and the residual's are aligned together.
template <typename T>
__device__ __forceinline__ void finish4(const ProdP& p, int64_t r, int64_t c, int n, float (&v)[4]) {
  const T* res = p.res ? (const T*)p.res + r * p.ldr + c : nullptr;
  T* y = (T*)p.y + r * p.ldy + c;
  float* pre = p.pre ? p.pre + r * p.cols + c : nullptr;
  constexpr uintptr_t A = 4 * sizeof(T) - 1;
  const bool wide = n == 4 && ((uintptr_t)y & A) == 0 && ((uintptr_t)res & A) == 0 && ((uintptr_t)pre & 15) == 0;
  float q[4] = {0.f, 0.f, 0.f, 0.f};
  if (res) {
    if (wide) {
      if constexpr (sizeof(T) == 2) {
        const uint2 w = *(const uint2*)res;
        q[0] = lo_bf16(w.x); q[1] = hi_bf16(w.x); q[2] = lo_bf16(w.y); q[3] = hi_bf16(w.y);
      } else {
        const float4 w = *(const float4*)res;
        q[0] = w.x; q[1] = w.y; q[2] = w.z; q[3] = w.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) q[i] = Elem<T>::load(res, i);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] += p.b && i < n ? p.b[c + i] : 0.f;
  if (pre) {
    if (wide) {
      *(float4*)pre = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) pre[i] = v[i];
    }
  }
  if (p.act != MTGNN_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act_(p.act, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] += q[i];
  if (wide) {
    if constexpr (sizeof(T) == 2) *(uint2*)y = make_uint2(cvt2_bf16(v[0], v[1]), cvt2_bf16(v[2], v[3]));
    else *(float4*)y = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) Elem<T>::store(y, i, v[i]);
  }
}

// A wave's WR x WC tiles of 16 x 16, rows from ra, columns from ca: sixteen rows at a time through LDS (s: the block's),
// so that lane l then has row l / (4 WC) of a few and four columns.  again(r, c, v): the value to take for v.
template <int WR, int WC, typename Y, class Again>
__device__ __forceinline__ void leave(const ProdP& p, const f32x4 (&acc)[WR][WC], float* lds, int64_t ra, int64_t ca,
                                      int64_t rows, int share, Again again) {
  constexpr int LD = 16 * WC + 4, LPR = 4 * WC;     // words of a row; lanes of a row
  const int lane = threadIdx.x & 63, fr = lane & 15, fg = lane >> 4;
  float* s = lds + (threadIdx.x >> 6) * 16 * LD;
  float* out = p.o + (p.split > 1 ? (int64_t)share * p.rows * p.cols : 0);
#pragma unroll
  for (int i = 0; i < WR; ++i) {
#pragma unroll
    for (int j = 0; j < WC; ++j) *(f32x4*)(s + fr * LD + 16 * j + 4 * fg) = acc[i][j];
    __syncthreads();
#pragma unroll 1
    for (int e = lane; e < 16 * LPR; e += 64) {
      const int64_t r = ra + 16 * i + e / LPR, c = ca + 4 * (e % LPR);
      if (r >= rows || c >= p.cols) continue;
      const f32x4 f = *(const f32x4*)(s + (e / LPR) * LD + 4 * (e % LPR));
      float v[4] = {f.x, f.y, f.z, f.w};
      const int n = (int)min((int64_t)4, p.cols - c);
      if (!(fabsf(f.x) + fabsf(f.y) + fabsf(f.z) + fabsf(f.w) < INFINITY)) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (u < n) v[u] = again(r, c + u, v[u]);
      }
      if (p.y) {
        finish4<Y>(p, r, c, n, v);
      } else if (n == 4 && ((uintptr_t)(out + r * p.ldo + c) & 15) == 0) {
        *(float4*)(out + r * p.ldo + c) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (u < n) out[r * p.ldo + c + u] = v[u];
      }
    }
    __syncthreads();
  }
}

// RF, CF: float32 operands; RK, CK: contiguous along k.  Y: the type of y.
template <bool RF, bool CF, bool RK, bool CK, int T>
__global__ __launch_bounds__(NT) void k_product(ProdP p) {
  constexpr int KS = T == 128 && (RF || CF) ? 32 : 64;
  constexpr int W = T / 32;                      // 16-wide tiles of a wave, each way
  using SR = Stage<RF, RK, T, KS>;
  using SC = Stage<CF, CK, T, KS>;
  using Y = std::conditional_t<CF, float, uint16_t>;
  constexpr int PLANE = T * KS / 2;              // words
  constexpr int WORDS = (SR::PL + SC::PL) * PLANE, OUT = 4 * 16 * (T / 2 + 4);   // words of the operands, of leave()
  constexpr int BUF = T == 128 && 2 * 4 * WORDS <= 65536 ? 2 : 1;   // two buffers (a barrier less) where they cost no block of a CU
  __shared__ __align__(16) uint32_t lds[BUF * WORDS > OUT ? BUF * WORDS : OUT];
  int64_t tr, tcol;
  int share;
  my_tile(p, tr, tcol, share);
  const int64_t rows = eff_count(p.rows, p.rows_dev), K = eff_count(p.K, p.K_dev);
  const int64_t r0 = tr * T, c0 = tcol * T;
  if (r0 >= rows) return;
  const int64_t per = cdiv(cdiv(K, KS), p.split) * KS;
  const int64_t kb = min(K, share * per), ke = min(K, kb + per);
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (wid >> 1) * (T / 2), wc = (wid & 1) * (T / 2), fr = lane & 15, fg = lane >> 4;
  f32x4 acc[W][W];
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int j = 0; j < W; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  SR a;
  SC b;
  a.at_rows(p.R, p.ldR, rows, r0);
  b.at_rows(p.C, p.ldC, p.cols, c0);
  if (kb < ke) {
    a.load(kb, ke);
    b.load(kb, ke);
  }
  for (int64_t k = kb; k < ke; k += KS) {
    uint32_t* sR = lds + (BUF > 1 && (k - kb) / KS % 2 ? WORDS : 0);
    uint32_t* sC = sR + SR::PL * PLANE;
    a.store(sR);
    b.store(sC);
    __syncthreads();
    if (k + KS < ke) {
      a.load(k + KS, ke);
      b.load(k + KS, ke);
    }
#pragma unroll
    for (int kk = 0; kk < KS / 32; ++kk) {
      bf16x8_t cf[W][SC::PL];
#pragma unroll
      for (int j = 0; j < W; ++j)
#pragma unroll
        for (int q = 0; q < SC::PL; ++q) cf[j][q] = SC::frag(sC, q, wc + 16 * j + fr, 4 * kk + fg);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        bf16x8_t rf[SR::PL];
#pragma unroll
        for (int q = 0; q < SR::PL; ++q) rf[q] = SR::frag(sR, q, wr + 16 * i + fr, 4 * kk + fg);
        const auto mul = [&](int qc, int qr) {
#pragma unroll
          for (int j = 0; j < W; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cf[j][qc], rf[qr], acc[i][j], 0, 0, 0);
        };
        if constexpr (RF && CF) {
          mul(1, 1);
          mul(2, 0);
          mul(0, 2);
          mul(1, 0);
          mul(0, 1);
        } else if constexpr (RF) {
          mul(0, 2);
          mul(0, 1);
        }
        mul(0, 0);
      }
    }
    if constexpr (BUF == 1) __syncthreads();
  }
  if constexpr (BUF > 1) __syncthreads();
  leave<W, W, Y>(p, acc, (float*)lds, r0 + wr, c0 + wc, rows, share, [&](int64_t r, int64_t c, float v) {
    if constexpr (RF || CF) {
      if (!(fabsf(v) < INFINITY)) return plain_sum<RF, CF, RK, CK>(p.R, p.ldR, p.C, p.ldC, r, c, kb, ke);
    }
    return v;
  });
}

// The same for bfloat16 operands that are contiguous along k, K a multiple of 64, where there are enough tiles of
// 256 x 256 for the card: 304 us in a row, 904 TFLOP/s, at 16,384 x 4,096 -> 2,048 with a residual (512 tiles; in a kernel
// trace 319, 305 at the least), 452 in tiles of 128; 67 against 82 us at 8,192 x 1,024 -> 2,048 with pre (256 tiles: one a
// CU, 96 MB written at its end).  What is left: waits for LDS, whose reads take 0.75 of the cycles of the matrix
// instructions, and the epilogue, which no other block of the CU hides.  Eight waves, 128 rows x 64 columns each: a matrix
// instruction needs 0.75 of the LDS bytes that it needs with 64 x 64.  Rows go straight to LDS, lane l of a load to unit
// l % 8 of row l / 8; the units' swizzle is in the address that the lane reads.  Two buffers, which are two objects, so that
// the compiler knows that the reads of one do not wait for the loads into the other; a step's loads are a whole step's work
// ahead.
constexpr int BIG = 256, BIG_KS = 64;
__global__ __launch_bounds__(512, 2) void k_product_big(ProdP p) {
  constexpr int WR = 8, WC = 4, OP = BIG * BIG_KS / 2;   // words of an operand's tile
  __shared__ __align__(1024) uint32_t bufA[2 * OP], bufB[2 * OP];
  int64_t tr, tcol;
  int share;
  my_tile(p, tr, tcol, share);
  const int64_t rows = eff_count(p.rows, p.rows_dev), K = p.K;
  const int64_t r0 = tr * BIG, c0 = tcol * BIG;
  if (r0 >= rows) return;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (wid >> 2) * 128, wc = (wid & 3) * 64, fr = lane & 15, fg = lane >> 4;
  // this wave's loads: rows 32 wid + 8 i + lane / 8 of each operand
  using S = Stage<false, true, BIG, BIG_KS>;
  const uint16_t* src[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 32 * wid + 8 * i + (lane >> 3), unit = (lane & 7) ^ S::turn(row);
    src[0][i] = (const uint16_t*)p.R + min(r0 + row, rows - 1) * p.ldR + 8 * unit;
    src[1][i] = (const uint16_t*)p.C + min(c0 + row, p.cols - 1) * p.ldC + 8 * unit;
  }
  typedef __attribute__((address_space(3))) void* lds_ptr;
  const auto fill = [&](uint32_t* buf, int64_t k) {
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_amdgcn_global_load_lds((void*)(src[o][i] + k), (lds_ptr)(buf + o * OP + (32 * wid + 8 * i) * (BIG_KS / 2)),
                                         16, 0, 0);
  };
  f32x4 acc[WR][WC];
#pragma unroll
  for (int i = 0; i < WR; ++i)
#pragma unroll
    for (int j = 0; j < WC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto multiply = [&](const uint32_t* buf) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8_t cf[WC];
#pragma unroll
      for (int j = 0; j < WC; ++j) cf[j] = S::frag(buf + OP, 0, wc + 16 * j + fr, 4 * kk + fg);
#pragma unroll
      for (int i = 0; i < WR; ++i) {
        const bf16x8_t rf = S::frag(buf, 0, wr + 16 * i + fr, 4 * kk + fg);
#pragma unroll
        for (int j = 0; j < WC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cf[j], rf, acc[i][j], 0, 0, 0);
      }
    }
  };
  const auto ready = [] {   // this wave's loads have arrived and its reads are done, then everybody's
    asm volatile("" ::: "memory");        // reads of LDS stay on their side
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  fill(bufA, 0);
  const int steps = (int)(K / BIG_KS);
  int step = 0;
  for (; step + 1 < steps; step += 2) {
    ready();
    fill(bufB, (int64_t)(step + 1) * BIG_KS);
    multiply(bufA);
    ready();
    if (step + 2 < steps) fill(bufA, (int64_t)(step + 2) * BIG_KS);
    multiply(bufB);
  }
  if (step < steps) {
    ready();
    multiply(bufA);
  }
  __syncthreads();
  leave<WR, WC, uint16_t>(p, acc, (float*)bufA, r0 + wr, c0 + wc, rows, 0, [](int64_t, int64_t, float v) { return v; });
}

// The sums of the shares of a split product, and what is left of the call.
template <typename Y>
__global__ __launch_bounds__(256) void k_product_sum(ProdP p, const float* part, int64_t total) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= total) return;
  const int64_t r = e / p.cols, c = e % p.cols;
  if (r >= eff_count(p.rows, p.rows_dev)) return;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < p.split; ++s) v[0] += part[s * total + e];
  if (p.y) finish4<Y>(p, r, c, 1, v);
  else p.o[r * p.ldo + c] = v[0];
}

// g = dy act'(pre), rows dense, and the column sums of each 16 rows (rows < n_rows; zeros without any).  A thread has V
// columns of 4 rows, all requested before the first is used.  Reading and writing bounds it: 33 us, 6.1 TB/s, at 8,192 x
// 2,048.  16 rows a block: 64 leave a quarter of the blocks, 46 us there and 25 us instead of 8 at 2,399 x 100; the
// column sums of the shares cost 12 us with 16 and 5 with 64.
constexpr int SLOPE_ROWS = 16;
template <int V>
__global__ __launch_bounds__(256) void k_linear_slope(const float* dy, int64_t lddy, const float* pre,
                                                      const int32_t* n_rows, int64_t max_rows, int n, int act,
                                                      float* g, float* part) {
  constexpr int M = SLOPE_ROWS / 4;
  __shared__ float s[4][64 * V];
  const int64_t rows = eff_count(max_rows, n_rows), cb = cdiv(n, 64 * V), blk = blockIdx.x / cb;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t c = ((blockIdx.x % cb) * 64 + lane) * V, r0 = blk * SLOPE_ROWS + wid * M;
  float sum[V];
#pragma unroll
  for (int u = 0; u < V; ++u) sum[u] = 0.f;
  if (c < n && r0 < rows) {
    const auto get = [](const float* p, float (&v)[V]) {
      if constexpr (V == 4) {
        const float4 f = *(const float4*)p;
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
      } else {
        v[0] = p[0];
      }
    };
    float d[M][V], q[M][V];
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int64_t r = min(r0 + i, rows - 1);
      get(dy + r * lddy + c, d[i]);
      if (act != MTGNN_ACT_NONE) get(pre + r * n + c, q[i]);
    }
#pragma unroll
    for (int i = 0; i < M; ++i) {
      if (r0 + i >= rows) break;
#pragma unroll
      for (int u = 0; u < V; ++u) {
        if (act != MTGNN_ACT_NONE) d[i][u] *= dact_(act, q[i][u]);
        sum[u] += d[i][u];
      }
      if (!g) continue;
      float* o = g + (r0 + i) * n + c;
      if constexpr (V == 4) *(float4*)o = make_float4(d[i][0], d[i][1], d[i][2], d[i][3]);
      else o[0] = d[i][0];
    }
  }
#pragma unroll
  for (int u = 0; u < V; ++u) s[wid][lane * V + u] = sum[u];
  __syncthreads();
  if (!part || wid) return;
#pragma unroll
  for (int u = 0; u < V; ++u)
    if (c < n) part[blk * n + c + u] = (s[0][lane * V + u] + s[1][lane * V + u]) + (s[2][lane * V + u] + s[3][lane * V + u]);
}

size_t al(size_t b) { return (b + 255) & ~size_t(255); }

// Tile side and blocks per tile's sum.  A tile of 128 takes half the operand traffic per product of one of 64, and
// needs two blocks a CU to hide a step's loads; with fewer than about 400 the smaller ones fill the card better.
// Sides of 128 against 64: 35 against 44 us at 1,092 tiles of 128, 147 against 207 at 512 (data gradients), 50
// against 46 at 272, 36 against 20 at 126.  Long sums with few tiles (weight gradients) take 128 and share the sum:
// 170 + 11 us against 280 (2,048 x 1,024 from 8,192 rows).  Shares have 128 k or more: 2,399 x 472 -> 100 takes 11 + 4.5 us
// in shares of 157, 13 + 5 in shares of 67, 22 without.
// Where these rules do not hold: they count tiles, not columns, so from 51,073 rows on a few outputs take the large tiles
// too (60,000 x 100 -> 32 24 us in float32, 16 in bfloat16; 40,000 rows 13 and 13); and forward calls of 4,096 inputs and more
// take 128 as weight gradients do, which costs those of few tiles up to half (1,000 x 8,192 -> 300 in bfloat16 34 against
// 24 us in tiles of 64, 300 x 4,096 -> 100 in float32 20 against 15) and gains with many (2,000 x 8,192 -> 600 63 against 87).
struct Plan {
  int T, split;
  int64_t tr, tc;
};
Plan plan(int64_t rows, int64_t cols, int64_t K) {
  Plan p;
  p.T = cdiv(rows, 128) * cdiv(cols, 128) >= 400 ? 128 : 64;
  if (p.T == 64 && rows > 64 && cols > 64 && K >= 4096) p.T = 128;   // long sums (dW): shares fill the card
  p.tr = cdiv(rows, p.T);
  p.tc = cdiv(cols, p.T);
  const int64_t t = std::max<int64_t>(1, p.tr * p.tc);   // (sizes are asked for no rows too)
  p.split = (int)std::max<int64_t>(1, std::min<int64_t>(t < 256 ? cdiv(512, t) : 1, K / 128));
  return p;
}
size_t split_bytes(int64_t rows, int64_t cols, int64_t K) {
  const Plan q = plan(rows, cols, K);
  return q.split > 1 ? al((size_t)q.split * rows * cols * 4) : 0;
}

// out = R C^T; the rest of p is set.
template <bool RF, bool CF, bool RK, bool CK>
mtgnn_status product(ProdP p, void* ws, hipStream_t s) {
  if constexpr (!RF && !CF && RK && CK) {
    if (p.aligned && p.K % BIG_KS == 0 && cdiv(p.rows, BIG) * cdiv(p.cols, BIG) >= 192) {
      p.tc = cdiv(p.cols, BIG);
      p.tiles = cdiv(p.rows, BIG) * p.tc;
      p.split = 1;
      TimedScope ts(site::Generic::name, s), tile("linear_256", s);
      k_product_big<<<(unsigned)p.tiles, 512, 0, s>>>(p);
      MTGNN_CHECK_LAUNCH("product_big");
      return MTGNN_OK;
    }
  }
  const Plan q = plan(p.rows, p.cols, p.K);
  p.tc = q.tc;
  p.tiles = q.tr * q.tc;
  p.split = q.split;
  const ProdP fin = p;
  if (q.split > 1) {
    p.o = (float*)ws;
    p.ldo = p.cols;
    p.y = nullptr;
  }
  const unsigned grid = (unsigned)(p.tiles * p.split);
  {
    TimedScope ts(site::Generic::name, s), tile(q.T == 128 ? "linear_128" : "linear_64", s);
    if (q.T == 128) k_product<RF, CF, RK, CK, 128><<<grid, NT, 0, s>>>(p);
    else k_product<RF, CF, RK, CK, 64><<<grid, NT, 0, s>>>(p);
  }
  MTGNN_CHECK_LAUNCH("product");
  if (q.split > 1) {
    const int64_t total = p.rows * p.cols;
    k_product_sum<std::conditional_t<CF, float, uint16_t>><<<(unsigned)cdiv(total, 256), 256, 0, s>>>(
        fin, (const float*)ws, total);
    MTGNN_CHECK_LAUNCH("product_sum");
  }
  return MTGNN_OK;
}

}  // namespace

// Work items of a launch are a 32-bit number.
bool linear_fits(const mtgnn_linear_dims* d, int64_t rows, bool back) {
  constexpr int64_t MAX = int64_t(1) << 32;
  const auto fits = [](int64_t r, int64_t c, int64_t K) {
    const Plan q = plan(r, c, K);
    return q.tr * q.tc * q.split * NT < MAX;
  };
  if (!back) return fits(rows, d->d_out, d->d_in);
  return fits(rows, d->d_in, d->d_out) && fits(d->d_out, d->d_in, rows) &&
         cdiv(rows, SLOPE_ROWS) * cdiv(d->d_out, 64) * 256 < MAX;
}

size_t linear_ws(const mtgnn_linear_dims* d, int64_t rows, bool back) {
  if (!back) return split_bytes(rows, d->d_out, d->d_in);
  const size_t g = al((size_t)rows * d->d_out * 4) + al((size_t)cdiv(rows, SLOPE_ROWS) * d->d_out * 4);
  return g + std::max(split_bytes(rows, d->d_in, d->d_out), split_bytes(d->d_out, d->d_in, rows));
}

mtgnn_status linear_impl(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const void* W,
                         const float* b, const void* res, int64_t ldr, const mtgnn_linear_dims* d, void* y,
                         int64_t ldy, float* pre, void* ws, size_t ws_bytes, hipStream_t s) {
  const bool bf = d->dtype == MTGNN_BF16;
  const int64_t per = bf ? 8 : 4;
  ProdP p{};
  p.R = x; p.ldR = ldx; p.C = W; p.ldC = d->d_in;
  p.rows = max_rows; p.cols = d->d_out; p.K = d->d_in; p.rows_dev = n_rows;
  p.aligned = ldx % per == 0 && d->d_in % per == 0 && ((uintptr_t)x | (uintptr_t)W) % 16 == 0;
  p.b = b; p.res = res; p.ldr = ldr; p.y = y; p.ldy = ldy; p.pre = pre; p.act = d->act;
  return bf ? product<false, false, true, true>(p, ws, s) : product<true, true, true, true>(p, ws, s);
}

mtgnn_status linear_bwd_impl(const float* dy, int64_t lddy, const float* pre, const void* x, int64_t ldx,
                             const int32_t* n_rows, int64_t max_rows, const void* W, const mtgnn_linear_dims* d,
                             float* dx, int64_t lddx, float* dW, float* db, void* ws, size_t ws_bytes, hipStream_t s) {
  const bool bf = d->dtype == MTGNN_BF16, direct = d->act == MTGNN_ACT_NONE;
  const int n = d->d_out;
  float* gbuf = (float*)ws;
  float* part = (float*)((char*)ws + al((size_t)max_rows * n * 4));
  void* rest = (char*)part + al((size_t)cdiv(max_rows, SLOPE_ROWS) * n * 4);
  const float* g = direct ? dy : gbuf;   // without an activation dy is the slope
  const int64_t ldg = direct ? lddy : n, blks = cdiv(max_rows, SLOPE_ROWS);
  if (!direct || db) {
    float *to = direct ? nullptr : gbuf, *sums = db ? part : nullptr;
    // Four columns a thread where that leaves four blocks a CU: 33 against 37 us (8,192 x 2,048); with fewer blocks one
    // column has the more waves: 4.7 against 8 us (2,399 x 100).
    if (blks * cdiv(n, 256) >= 1024 && n % 4 == 0 && lddy % 4 == 0 && ((uintptr_t)dy | (uintptr_t)pre | (uintptr_t)to) % 16 == 0)
      k_linear_slope<4><<<(unsigned)(blks * cdiv(n, 256)), 256, 0, s>>>(dy, lddy, pre, n_rows, max_rows, n, d->act, to, sums);
    else
      k_linear_slope<1><<<(unsigned)(blks * cdiv(n, 64)), 256, 0, s>>>(dy, lddy, pre, n_rows, max_rows, n, d->act, to, sums);
    MTGNN_CHECK_LAUNCH("linear_slope");
  }
  if (db) {
    k_sum_parts<<<(unsigned)cdiv(n, 16), 256, 0, s>>>(Seqs{}, 0, (int)blks, part, n, n, db, 0, nullptr, nullptr);
    MTGNN_CHECK_LAUNCH("linear_sum_parts");
  }
  if (dx) {
    ProdP p{};
    p.R = g; p.ldR = ldg; p.C = W; p.ldC = d->d_in;
    p.rows = max_rows; p.cols = d->d_in; p.K = n; p.rows_dev = n_rows;
    p.o = dx; p.ldo = lddx;
    MTGNN_TRY((bf ? product<true, false, true, false>(p, rest, s) : product<true, true, true, false>(p, rest, s)));
  }
  ProdP p{};
  p.R = g; p.ldR = ldg; p.C = x; p.ldC = ldx;
  p.rows = n; p.cols = d->d_in; p.K = max_rows; p.K_dev = n_rows;
  p.o = dW; p.ldo = d->d_in;
  return bf ? product<true, false, false, false>(p, rest, s) : product<true, true, false, false>(p, rest, s);
}

}  // namespace mtgnn
