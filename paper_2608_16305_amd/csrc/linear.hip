// Linear layer with bias, activation and residual, and its backward.
#include "gemm.h"
#include "ops.h"
#include "seq.h"

namespace mtgnn {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void k_linear_out(const float* pre, const T* res, int64_t ldr, const int32_t* n_rows,
                                                    int64_t max_rows, int n, int act, T* y, int64_t ldy) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, row = e / n;
  if (row >= eff_count(max_rows, n_rows)) return;
  const int64_t col = e % n;
  float v = act_(act, pre[row * n + col]);
  if (res) v += Elem<T>::load(res, row * ldr + col);
  Elem<T>::store(y, row * ldy + col, v);
}

__global__ __launch_bounds__(256) void k_linear_slope(const float* dy, int64_t lddy, const float* pre,
                                                      const int32_t* n_rows, int64_t max_rows, int n, int act,
                                                      float* g) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, row = e / n;
  if (row >= eff_count(max_rows, n_rows)) return;
  const int64_t col = e % n;
  const float d = dy[row * lddy + col];
  g[e] = act == MTGNN_ACT_NONE ? d : d * dact_(act, pre[e]);
}

size_t al(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace

size_t linear_ws(const mtgnn_linear_dims* d, int64_t rows, bool back) {
  const size_t m = al((size_t)rows * d->d_out * 4);
  return back ? m + al(linear_dw_ws_bytes(rows, d->d_out, d->d_in)) : m;
}

mtgnn_status linear_impl(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const void* W,
                         const float* b, const void* res, int64_t ldr, const mtgnn_linear_dims* d, void* y,
                         int64_t ldy, float* pre, void* ws, size_t ws_bytes, hipStream_t s) {
  float* p = pre ? pre : (float*)ws;
  MTGNN_TRY((linear_fwd(x, d->dtype, ldx, W, d->dtype, d->d_in, b, p, d->d_out, max_rows, n_rows, d->d_out, d->d_in,
                        false, s)));
  const unsigned grid = (unsigned)cdiv(max_rows * d->d_out, 256);
  if (d->dtype == MTGNN_BF16)
    k_linear_out<uint16_t><<<grid, 256, 0, s>>>(p, (const uint16_t*)res, ldr, n_rows, max_rows, d->d_out, d->act,
                                                (uint16_t*)y, ldy);
  else
    k_linear_out<float><<<grid, 256, 0, s>>>(p, (const float*)res, ldr, n_rows, max_rows, d->d_out, d->act, (float*)y,
                                             ldy);
  MTGNN_CHECK_LAUNCH("linear_out");
  return MTGNN_OK;
}

mtgnn_status linear_bwd_impl(const float* dy, int64_t lddy, const float* pre, const void* x, int64_t ldx,
                             const int32_t* n_rows, int64_t max_rows, const void* W, const mtgnn_linear_dims* d,
                             float* dx, int64_t lddx, float* dW, float* db, void* ws, size_t ws_bytes, hipStream_t s) {
  float* g = (float*)ws;
  const size_t m = al((size_t)max_rows * d->d_out * 4);
  k_linear_slope<<<(unsigned)cdiv(max_rows * d->d_out, 256), 256, 0, s>>>(dy, lddy, pre, n_rows, max_rows, d->d_out,
                                                                         d->act, g);
  MTGNN_CHECK_LAUNCH("linear_slope");
  if (dx)
    MTGNN_TRY((linear_dx(g, d->d_out, W, d->dtype, d->d_in, dx, lddx, max_rows, n_rows, d->d_out, d->d_in, false, s)));
  return linear_dw(g, d->d_out, x, d->dtype, ldx, dW, d->d_in, max_rows, n_rows, d->d_out, d->d_in, (char*)ws + m,
                   ws_bytes - m, s, db);
}

}  // namespace mtgnn
