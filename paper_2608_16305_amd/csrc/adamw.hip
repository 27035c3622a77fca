// An AdamW step (decoupled weight decay) over any number of tensors:
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),
// with m and v in float32, or in 8 bits: e4m3 codes of m and of sqrt(v), times a power of two for each 32 elements.
//
// Bound by memory: 28 bytes an element (30 with a bfloat16 copy), 16 in 8 bits (18).  Tensors of all sizes go in one launch
// (TENSORS of them, their descriptions being kernel arguments): a block finds its tensor by the first block of each.
//
// The 8-bit states hold the root of v, whose range is half as many binades: e4m3 has 2^17 between its largest and smallest
// number, so a v 2^-35 of its block's largest is still held.  They are formed in 64 bits and rounded once (m + (1 - b1) g
// near the border of two codes is decided as the formula says, whatever float32 would make of it; away from one float32
// decides, which is half of the instructions); a root that is not zero never becomes zero, for m / sqrt(v) has no bound there.
// The parameter's step uses m and v before that rounding.
#include <algorithm>
#include <cmath>

#include "ops.h"
#include "words.h"

namespace mtgnn {

namespace {

constexpr int NT = 256, PER = 4;   // threads; elements of a vector
constexpr int TENSORS = 40;

struct Set {
  mtgnn_adamw_tensor t[TENSORS];
  uint32_t first[TENSORS + 1];   // first block of each
  int count;
};

struct Coef {
  double b1, b2;                 // (1 - b is formed from them in double)
  float lr, eps, ibc1, ibc2;     // 1 / (1 - b^t)
  const int32_t* step;           // device step count, or NULL: ibc1 and ibc2 hold
};

typedef uint32_t word_at1 __attribute__((aligned(1)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ double pow_int(double b, int t) {   // by squares
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// e4m3: sign, four bits of exponent (bias 7), three of mantissa; 448 the largest, 2^-9 the least; no infinity, 0x7f is NaN.
// The nearest code (ties to even) of a >= 0 that is at most 448; of what is not finite NaN.
__device__ __attribute__((noinline)) uint32_t exact_code(double a) {
  if (!(a < INFINITY)) return 0x7fu;
  if (a < 0.015625) return (uint32_t)rint(a * 512.0);   // multiples of 2^-9 below 2^-6 (8 of them: 2^-6)
  const uint64_t u = (uint64_t)__double_as_longlong(a);
  return (uint32_t)((u + 0xffffffffffffull + (u >> 49 & 1)) >> 49) - (1016u << 3);
}
// Whether a float32 value that is off by a few units in its last place may be on the wrong side of a border of two codes: the 20
// bits behind a code's are near a half.  (Below 2^-6 the codes are 2^-9 apart: as far as they are from 2^-6 on.)
__device__ __forceinline__ bool near_border(float a) {
  const uint32_t u = __float_as_uint(a < 0.015625f ? a + 0.015625f : a);
  return (u & 0xfffffu) - 0x7fff8u <= 0x10u || !(a < 448.f);
}
// The biased exponent e of a block whose largest magnitude is `top`: top <= 448 2^(e - 127), the least such e.
__device__ __forceinline__ int exact_exponent(double top) {
  if (!(top > 0.0)) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(top);
  const int x = (int)(u >> 52) - 1022;   // top = f 2^x, f in [0.5, 1) (a subnormal one: x = -1022)
  const int e = x - 9 + ((u & 0xfffffffffffffull) > 0xc000000000000ull);
  return min(max(e, -127), 127) + 127;
}
__device__ __forceinline__ int block_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  return min(max((int)(u >> 23) - 126 - 9 + (int)((u & 0x7fffffu) > 0x600000u) + 127, 0), 254);
}
__device__ __forceinline__ bool exponent_unsure(float top) {   // near 448 times a power of two
  return (__float_as_uint(top) & 0x7fffffu) - 0x5ffff8u <= 0x10u;
}
__device__ __forceinline__ double pow2(int e) { return __longlong_as_double((long long)(e + 1023) << 52); }   // |e| < 1023
__device__ __forceinline__ float pow2f(int e) {   // -127 .. 127
  return e > -127 ? __uint_as_float((uint32_t)(e + 127) << 23) : __uint_as_float(0x400000u);
}
__device__ __forceinline__ float max8(float v) {   // over eight lanes
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ double max8(double v) {
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) v = fmax(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ float finite(float v) { return v < INFINITY ? v : 0.f; }   // (v >= 0 or NaN)
__device__ __forceinline__ double finite(double v) { return v < INFINITY ? v : 0.0; }

// a x + b y, each operation rounded: a sum may be meant to lie on a border (0.9 times a code is one now and then), and is there
// only if its products are what 64 bits make of them.
__device__ __forceinline__ double sum64(double a, double x, double b, double y) {
#pragma clang fp contract(off)
  const double p = a * x, q = b * y;
  return p + q;
}

// The codes and the exponent of four elements' magnitudes, x in 64 bits and f as float32 (of the block's eight lanes).
// Decided in float32; what is near a border, from x itself (root: from its root).
template <bool ROOT>
__device__ __forceinline__ void encode(const double (&x)[PER], const float (&f)[PER], uint32_t& codes, int& exponent) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) top = fmaxf(top, finite(f[j]));
  top = max8(top);
  exponent = block_exponent(top);
  if (__any(exponent_unsure(top))) {
    double t = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) t = fmax(t, finite(fabs(x[j])));
    t = max8(t);
    exponent = exact_exponent(ROOT ? sqrt(t) : t);
  }
  const float by = pow2f(127 - exponent);
  float a[PER];
  bool unsure = false;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    a[j] = f[j] * by;
    unsure |= near_border(a[j]);
  }
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], 0, false);
  c = __builtin_amdgcn_cvt_pk_fp8_f32(a[2], a[3], c, true);
  codes = (uint32_t)c;
  if (__any(unsure)) {
    uint32_t sure = 0u;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      sure |= (near_border(a[j]) ? exact_code((ROOT ? sqrt(x[j]) : fabs(x[j])) * pow2(127 - exponent)) : codes >> 8 * j & 255u) << 8 * j;
    codes = sure;
  }
}

// Vectors of a thread, all requested before the first is used.  Few, and many waves instead, which hide the arithmetic of one by
// the loads of others: 537 us with one, 587 with two and 728 with four in 8 bits (151M elements, 5.1 TB/s); 394, 404 and 416 with
// two, four and eight in 32 (69M, 5.2 TB/s).
template <bool BITS8>
constexpr int VECTORS = BITS8 ? 1 : 2;

template <bool BITS8>
__global__ __launch_bounds__(NT) void k_adamw(Set a, Coef c) {
  constexpr int N = VECTORS<BITS8>, TILE = NT * PER * N;
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.first[mid] <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const mtgnn_adamw_tensor t = a.t[lo];
  const int64_t e0 = (int64_t)(blockIdx.x - a.first[lo]) * TILE + threadIdx.x * PER;
  float ibc1 = c.ibc1, ibc2 = c.ibc2;
  if (c.step) {
    const int n = *c.step;
    ibc1 = (float)(1.0 / (1.0 - pow_int(c.b1, n)));
    ibc2 = (float)(1.0 / (1.0 - pow_int(c.b2, n)));
  }
  const float keep = c.lr * t.decay, sbc2 = sqrtf(ibc2);
  const double o1 = 1.0 - c.b1, o2 = 1.0 - c.b2;
  float p[N][PER], g[N][PER], m[N][PER], v[N][PER];
  uint32_t mc[N], vc[N];
  int me[N], ve[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t e = e0 + i * NT * PER;
    const int n = (int)min((int64_t)PER, t.n - e);
    mc[i] = vc[i] = 0u;
    me[i] = ve[i] = 0;
    if (n <= 0) continue;
    load_some((const float*)t.param + e, n, p[i]);
    load_some(t.grad + e, n, g[i]);
    if constexpr (BITS8) {
      if (n == PER) {
        mc[i] = *(const word_at1*)((const uint8_t*)t.m + e);
        vc[i] = *(const word_at1*)((const uint8_t*)t.v + e);
      } else {
        for (int j = 0; j < n; ++j) {
          mc[i] |= (uint32_t)((const uint8_t*)t.m)[e + j] << 8 * j;
          vc[i] |= (uint32_t)((const uint8_t*)t.v)[e + j] << 8 * j;
        }
      }
      me[i] = t.m_exp[e >> 5];
      ve[i] = t.v_exp[e >> 5];
    } else {
      load_some((const float*)t.m + e, n, m[i]);
      load_some((const float*)t.v + e, n, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t e = e0 + i * NT * PER;
    const int n = (int)min((int64_t)PER, t.n - e);
    if constexpr (BITS8) {
      double md[PER], vd[PER];
      const float ms = pow2f(me[i] - 127), vs = pow2f(ve[i] - 127);
      float am[PER], mo[PER], ro[PER];
      const f32x2 m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mc[i], false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mc[i], true);
      const f32x2 r01 = __builtin_amdgcn_cvt_pk_f32_fp8(vc[i], false), r23 = __builtin_amdgcn_cvt_pk_f32_fp8(vc[i], true);
      mo[0] = m01.x; mo[1] = m01.y; mo[2] = m23.x; mo[3] = m23.y;
      ro[0] = r01.x; ro[1] = r01.y; ro[2] = r23.x; ro[3] = r23.y;
#pragma unroll
      for (int j = 0; j < PER; ++j) {   // (codes times their units are exact)
        const double r = (double)(ro[j] * vs), x = j < n ? (double)g[i][j] : 0.0;
        md[j] = sum64(c.b1, (double)(mo[j] * ms), o1, x);
        vd[j] = sum64(c.b2, r * r, o2, x * x);
        m[i][j] = (float)md[j];
        am[j] = fabsf(m[i][j]);
        v[i][j] = (float)__builtin_amdgcn_sqrt(vd[j]);   // (the instruction's root: within a few float32 units)
      }
      encode<false>(md, am, mc[i], me[i]);
      encode<true>(vd, v[i], vc[i], ve[i]);
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (md[j] < 0.0) mc[i] |= 0x80u << 8 * j;
        if (vd[j] > 0.0 && (vc[i] >> 8 * j & 255u) == 0u) vc[i] |= 1u << 8 * j;
      }
    }
    if (n <= 0) continue;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if constexpr (!BITS8) {
        m[i][j] = (float)c.b1 * m[i][j] + (float)o1 * g[i][j];
        v[i][j] = (float)c.b2 * v[i][j] + (float)o2 * (g[i][j] * g[i][j]);
      }
      // (v: in 8 bits its root already)
      const float root = BITS8 ? v[i][j] * sbc2 : sqrtf(v[i][j] * ibc2);
      p[i][j] = (p[i][j] - keep * p[i][j]) - c.lr * (m[i][j] * ibc1) / (root + c.eps);
    }
    store_some(t.param + e, n, p[i]);
    if (t.shadow) store_some(t.shadow + e, n, p[i]);
    if constexpr (BITS8) {
      if (n == PER) {
        *(word_at1*)((uint8_t*)t.m + e) = mc[i];
        *(word_at1*)((uint8_t*)t.v + e) = vc[i];
      } else {
        for (int j = 0; j < n; ++j) {
          ((uint8_t*)t.m)[e + j] = (uint8_t)(mc[i] >> 8 * j);
          ((uint8_t*)t.v)[e + j] = (uint8_t)(vc[i] >> 8 * j);
        }
      }
      if ((e & 31) == 0) {
        t.m_exp[e >> 5] = (uint8_t)me[i];
        t.v_exp[e >> 5] = (uint8_t)ve[i];
      }
    } else {
      store_some((float*)t.m + e, n, m[i]);
      store_some((float*)t.v + e, n, v[i]);
    }
  }
}

}  // namespace

mtgnn_status adamw_impl(const mtgnn_adamw_tensor* tensors, int64_t n, const mtgnn_adam_config* cfg, const int32_t* step,
                        hipStream_t s) {
  Coef c;
  c.b1 = cfg->beta1;
  c.b2 = cfg->beta2;
  c.lr = (float)cfg->lr;
  c.eps = (float)cfg->eps;
  c.ibc1 = (float)(1.0 / (1.0 - std::pow(cfg->beta1, (double)cfg->t)));
  c.ibc2 = (float)(1.0 / (1.0 - std::pow(cfg->beta2, (double)cfg->t)));
  c.step = step;
  // both kinds of states may be in one call: a launch takes tensors of one kind
  for (int kind = 0; kind < 2; ++kind) {
    Set a{};
    int64_t blocks = 0;
    const auto launch = [&]() -> mtgnn_status {
      if (a.count == 0) return MTGNN_OK;
      a.first[a.count] = (uint32_t)blocks;
      if (kind) k_adamw<true><<<(unsigned)blocks, NT, 0, s>>>(a, c);
      else k_adamw<false><<<(unsigned)blocks, NT, 0, s>>>(a, c);
      MTGNN_CHECK_LAUNCH("adamw");
      a.count = 0;
      blocks = 0;
      return MTGNN_OK;
    };
    for (int64_t i = 0; i < n; ++i) {
      if (tensors[i].n == 0 || (tensors[i].m_exp != nullptr) != (kind == 1)) continue;
      const int64_t need = cdiv(tensors[i].n, NT * PER * (kind ? VECTORS<true> : VECTORS<false>));
      if (a.count == TENSORS || blocks + need > (int64_t(1) << 24) - 1) MTGNN_TRY(launch());
      a.t[a.count] = tensors[i];
      a.first[a.count++] = (uint32_t)blocks;
      blocks += need;
    }
    MTGNN_TRY(launch());
  }
  return MTGNN_OK;
}

}  // namespace mtgnn
