// Sixteen bytes, and fewer, of elements at any element's address: global loads and stores take it, so a row of an odd length
// or a column range of a wider matrix is read and written as wide as an aligned one.
#pragma once

#include "bf16_split.h"

namespace mtgnn {

typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));

// V elements of T from p on, as floats; n of them (n < V: one by one, the others are 0).
template <typename T, int V>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[V]) {
  if (n >= V) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const f32x4_at4 w = *(const f32x4_at4*)(p + i);
        v[i] = w.x; v[i + 1] = w.y; v[i + 2] = w.z; v[i + 3] = w.w;
      }
    } else if constexpr (V == 4) {
      const u32x2_at2 w = *(const u32x2_at2*)p;
      v[0] = lo_bf16(w.x); v[1] = hi_bf16(w.x); v[2] = lo_bf16(w.y); v[3] = hi_bf16(w.y);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 8) {
        const u32x4_at2 w = *(const u32x4_at2*)(p + i);
        v[i] = lo_bf16(w.x); v[i + 1] = hi_bf16(w.x); v[i + 2] = lo_bf16(w.y); v[i + 3] = hi_bf16(w.y);
        v[i + 4] = lo_bf16(w.z); v[i + 5] = hi_bf16(w.z); v[i + 6] = lo_bf16(w.w); v[i + 7] = hi_bf16(w.w);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < n ? Elem<T>::load(p, i) : 0.f;
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[V]) {
  if (n >= V) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; i += 4) *(f32x4_at4*)(p + i) = f32x4_at4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else if constexpr (V == 4) {
      *(u32x2_at2*)p = u32x2_at2{cvt2_bf16(v[0], v[1]), cvt2_bf16(v[2], v[3])};
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 8)
        *(u32x4_at2*)(p + i) = u32x4_at2{cvt2_bf16(v[i], v[i + 1]), cvt2_bf16(v[i + 2], v[i + 3]),
                                         cvt2_bf16(v[i + 4], v[i + 5]), cvt2_bf16(v[i + 6], v[i + 7])};
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) Elem<T>::store(p, i, v[i]);
  }
}

}  // namespace mtgnn
