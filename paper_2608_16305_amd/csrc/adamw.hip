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
// near the border of two codes is decided as the formula says, whatever float32 would make of it); a root that is
// not zero never becomes zero, for m / sqrt(v) has no bound there.  The parameter's step uses m and v before that rounding.
#include <algorithm>
#include <cmath>

#include "ops.h"
#include "words.h"

namespace mtgnn {

namespace {

constexpr int NT = 256, PER = 4, TILE = NT * PER * 4;   // elements of a block: four vectors of four a thread
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

__device__ __forceinline__ double pow_int(double b, int t) {   // by squares
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// e4m3: sign, four bits of exponent (bias 7), three of mantissa; 448 the largest, 2^-9 the least; no infinity, 0x7f is NaN.
__device__ __forceinline__ float of_e4m3(uint32_t c) {
  return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
}
// The nearest code (ties to even) of a >= 0 that is at most 448.
__device__ __forceinline__ uint32_t to_e4m3(double a) {
  if (!(a >= 0.015625)) return a != a ? 0x7fu : (uint32_t)rint(a * 512.0);   // multiples of 2^-9 below 2^-6 (8 of them: 2^-6)
  const uint64_t u = (uint64_t)__double_as_longlong(a);
  const uint32_t c = (uint32_t)((u + 0xffffffffffffull + (u >> 49 & 1)) >> 49) - (1016u << 3);
  return c < 0x7fu ? c : 0x7fu;
}
// The biased exponent e of a block whose largest magnitude is `top`: top <= 448 2^(e - 127), the least such e.
__device__ __forceinline__ int block_exponent(double top) {
  if (!(top > 0.0)) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(top);
  const int x = (int)(u >> 52) - 1022;   // top = f 2^x, f in [0.5, 1) (a subnormal one: x = -1022)
  const int e = x - 9 + ((u & 0xfffffffffffffull) > 0xc000000000000ull);
  return min(max(e, -127), 127) + 127;
}
__device__ __forceinline__ double pow2(int e) { return __longlong_as_double((long long)(e + 1023) << 52); }   // |e| < 1023
__device__ __forceinline__ double max8(double v) {   // over eight lanes; NaN stays out (its codes say it)
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) v = fmax(v, __shfl_xor(v, o, 64));
  return v;
}

template <bool BITS8>
__global__ __launch_bounds__(NT) void k_adamw(Set a, Coef c) {
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
  const float keep = c.lr * t.decay;
  const double o1 = 1.0 - c.b1, o2 = 1.0 - c.b2;
  float p[4][PER], g[4][PER], m[4][PER], v[4][PER];
  uint32_t mc[4], vc[4];
  int me[4], ve[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
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
  for (int i = 0; i < 4; ++i) {
    const int64_t e = e0 + i * NT * PER;
    const int n = (int)min((int64_t)PER, t.n - e);
    if constexpr (BITS8) {
      double md[PER], vd[PER], mt = 0.0, vt = 0.0;
      const double ms = pow2(me[i] - 127), vs = pow2(ve[i] - 127);
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const double r = (double)of_e4m3(vc[i] >> 8 * j & 255u) * vs, x = j < n ? (double)g[i][j] : 0.0;
        md[j] = c.b1 * ((double)of_e4m3(mc[i] >> 8 * j & 255u) * ms) + o1 * x;
        vd[j] = c.b2 * (r * r) + o2 * (x * x);
        mt = fmax(mt, fabs(md[j]) < INFINITY ? fabs(md[j]) : 0.0);   // (what is infinite has a code of its own: NaN)
        vt = fmax(vt, vd[j] < INFINITY ? vd[j] : 0.0);
        m[i][j] = (float)md[j];
        v[i][j] = (float)vd[j];
      }
      me[i] = block_exponent(max8(mt));
      ve[i] = block_exponent(sqrt(max8(vt)));
      const double mi = pow2(127 - me[i]), vi = pow2(127 - ve[i]);
      mc[i] = vc[i] = 0u;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const uint32_t mq = to_e4m3(fabs(md[j]) * mi) | (md[j] < 0.0 ? 0x80u : 0u);
        uint32_t vq = to_e4m3(sqrt(vd[j]) * vi);
        if (vq == 0u && vd[j] > 0.0) vq = 1u;
        mc[i] |= mq << 8 * j;
        vc[i] |= vq << 8 * j;
      }
    }
    if (n <= 0) continue;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if constexpr (!BITS8) {
        m[i][j] = (float)c.b1 * m[i][j] + (float)o1 * g[i][j];
        v[i][j] = (float)c.b2 * v[i][j] + (float)o2 * (g[i][j] * g[i][j]);
      }
      p[i][j] = (p[i][j] - keep * p[i][j]) - c.lr * (m[i][j] * ibc1) / (sqrtf(v[i][j] * ibc2) + c.eps);
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
      const int64_t need = cdiv(tensors[i].n, TILE);
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
