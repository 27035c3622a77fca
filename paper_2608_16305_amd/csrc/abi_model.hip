// C ABI of the operators of a model over all nodes: argument validation (host only, before any HIP call) and dispatch.
#include <algorithm>
#include <cmath>

#include "abi_check.h"

using namespace mtgnn;

namespace {

mtgnn_status check_embedding(const mtgnn_embedding_dims* d) {
  if (!d) return fail(MTGNN_EINVAL, "dims is NULL");
  if (!dtype_ok(d->dtype)) return fail(MTGNN_EUNSUPPORTED, "dtype");
  if (d->n <= 0 || d->d <= 0) return fail(MTGNN_EINVAL, "non-positive dimension");
  if (d->n >= MAX_ROWS || d->d > MAX_WIDTH) return fail(MTGNN_EUNSUPPORTED, "n or d too large");
  if (!std::isfinite(d->scale)) return fail(MTGNN_EINVAL, "scale is not finite");
  return MTGNN_OK;
}

mtgnn_status check_norm(const mtgnn_norm_dims* d) {
  if (!d) return fail(MTGNN_EINVAL, "dims is NULL");
  if (!dtype_ok(d->dtype)) return fail(MTGNN_EUNSUPPORTED, "dtype");
  if (d->d <= 0) return fail(MTGNN_EINVAL, "non-positive dimension");
  if (d->d > MAX_WIDTH) return fail(MTGNN_EUNSUPPORTED, "d > 2^20");
  if (!std::isfinite(d->eps) || d->eps < 0.f) return fail(MTGNN_EINVAL, "eps is negative or not finite");
  return MTGNN_OK;
}

mtgnn_status check_loss(const mtgnn_loss_dims* d) {
  if (!d) return fail(MTGNN_EINVAL, "dims is NULL");
  if (!dtype_ok(d->dtype)) return fail(MTGNN_EUNSUPPORTED, "dtype");
  if (d->n <= 0 || d->d <= 0) return fail(MTGNN_EINVAL, "non-positive dimension");
  if (d->n >= MAX_ROWS || d->d > MAX_WIDTH) return fail(MTGNN_EUNSUPPORTED, "n or d too large");
  return MTGNN_OK;
}

// Written and read two floats at a time.
mtgnn_status check_stats(const float* stats) {
  return (uintptr_t)stats % 8 ? fail(MTGNN_EINVAL, "stats is not 8-byte aligned") : MTGNN_OK;
}

// A block of `threads` to each row.
mtgnn_status check_blocks(int64_t rows, int64_t threads, const char* what) { return check_items(rows, threads, what); }

}  // namespace

extern "C" {

mtgnn_status mtgnn_embedding(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const void* table,
                             const mtgnn_embedding_dims* d, void* y, int64_t ldy, hipStream_t stream) {
  MTGNN_TRY(check_embedding(d));
  MTGNN_TRY(check_rows(max_rows, 1));
  if (max_rows == 0) return MTGNN_OK;
  REQ(ids, "ids");
  REQ(table, "table");
  REQ(y, "y");
  STRIDE(ldy, d->d, "ldy");
  if (!embed_fits(d, max_rows, false)) return fail(MTGNN_EUNSUPPORTED, "max_rows times d");
  const int64_t e = bytes_of(d->dtype);
  if (overlap(Rows{table, d->n * d->d * e, d->n * d->d * e}, Rows{y, ((max_rows - 1) * ldy + d->d) * e, ((max_rows - 1) * ldy + d->d) * e}, 1))
    return fail(MTGNN_EINVAL, "y overlaps the table");
  return embed_impl(ids, n_rows, max_rows, table, d, y, ldy, stream);
}

size_t mtgnn_embedding_ws_bytes(const mtgnn_embedding_dims* d, int64_t max_rows) {
  if (check_embedding(d) != MTGNN_OK || check_rows(max_rows, 1) != MTGNN_OK) return 0;
  return embed_ws(d, max_rows);
}

mtgnn_status mtgnn_embedding_bwd(const int32_t* ids, const int32_t* n_rows, int64_t max_rows, const float* dy, int64_t lddy,
                                 const mtgnn_embedding_dims* d, float* dtable, void* ws, size_t ws_bytes,
                                 hipStream_t stream) {
  MTGNN_TRY(check_embedding(d));
  MTGNN_TRY(check_rows(max_rows, 1));
  if (max_rows == 0) return fail(MTGNN_EINVAL, "max_rows == 0 (no row: the gradient is zero; skip the call)");
  REQ(ids, "ids");
  REQ(dy, "dy");
  REQ(dtable, "dtable");
  STRIDE(lddy, d->d, "lddy");
  if (!embed_fits(d, max_rows, true)) return fail(MTGNN_EUNSUPPORTED, "n or max_rows times d");
  if (ws_bytes < embed_ws(d, max_rows)) return fail(MTGNN_EWORKSPACE, "embedding_bwd ws");
  REQ(ws, "ws");
  MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  const int64_t to = d->n * d->d * 4, from = ((max_rows - 1) * lddy + d->d) * 4;
  if (overlap(Rows{dtable, to, to}, Rows{dy, from, from}, 1)) return fail(MTGNN_EINVAL, "dtable overlaps dy");
  return embed_bwd_impl(ids, n_rows, max_rows, dy, lddy, d, dtable, ws, stream);
}

mtgnn_status mtgnn_layer_norm(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const float* gamma,
                              const float* beta, const mtgnn_norm_dims* d, void* y, int64_t ldy, float* stats,
                              hipStream_t stream) {
  MTGNN_TRY(check_norm(d));
  MTGNN_TRY(check_rows(max_rows, d->d));
  if (max_rows == 0) return MTGNN_OK;
  REQ(x, "x");
  REQ(y, "y");
  STRIDE(ldx, d->d, "ldx");
  STRIDE(ldy, d->d, "ldy");
  MTGNN_TRY(check_stats(stats));
  MTGNN_TRY(check_blocks(max_rows, norm_threads(d), "max_rows"));
  const int64_t e = bytes_of(d->dtype), w = d->d * e;
  if ((x != y || ldx != ldy || stats) && overlap(Rows{x, ldx * e, w}, Rows{y, ldy * e, w}, max_rows))
    return fail(MTGNN_EINVAL, "y overlaps x");
  return norm_impl(x, ldx, n_rows, max_rows, gamma, beta, d, y, ldy, stats, stream);
}

size_t mtgnn_layer_norm_ws_bytes(const mtgnn_norm_dims* d, int64_t max_rows) {
  if (check_norm(d) != MTGNN_OK || check_rows(max_rows, d->d) != MTGNN_OK) return 0;
  return norm_ws(d, max_rows);
}

mtgnn_status mtgnn_layer_norm_bwd(const float* dy, int64_t lddy, const void* x, int64_t ldx, const float* stats,
                                  const int32_t* n_rows, int64_t max_rows, const float* gamma, const float* past, int64_t ldp,
                                  const mtgnn_norm_dims* d, float* dx, int64_t lddx, float* dgamma, float* dbeta, void* ws,
                                  size_t ws_bytes, hipStream_t stream) {
  MTGNN_TRY(check_norm(d));
  MTGNN_TRY(check_rows(max_rows, d->d));
  if (max_rows == 0) return fail(MTGNN_EINVAL, "max_rows == 0 (no row: every gradient is zero; skip the call)");
  REQ(dy, "dy");
  REQ(x, "x");
  REQ(stats, "stats");
  REQ(dx, "dx");
  STRIDE(lddy, d->d, "lddy");
  STRIDE(ldx, d->d, "ldx");
  STRIDE(lddx, d->d, "lddx");
  if (past) STRIDE(ldp, d->d, "ldp");
  MTGNN_TRY(check_stats(stats));
  MTGNN_TRY(check_blocks(max_rows, norm_threads(d), "max_rows"));
  if (dgamma || dbeta) {
    if (ws_bytes < norm_ws(d, max_rows)) return fail(MTGNN_EWORKSPACE, "layer_norm_bwd ws");
    REQ(ws, "ws");
    MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  }
  const int64_t e = bytes_of(d->dtype), w = (int64_t)d->d * 4;
  const Rows to{dx, lddx * 4, w};
  if ((dx != dy || lddx != lddy) && overlap(to, Rows{dy, lddy * 4, w}, max_rows)) return fail(MTGNN_EINVAL, "dx overlaps dy");
  if ((dx != past || lddx != ldp) && overlap(to, Rows{past, ldp * 4, w}, max_rows)) return fail(MTGNN_EINVAL, "dx overlaps past");
  if (overlap(to, Rows{x, ldx * e, d->d * e}, max_rows)) return fail(MTGNN_EINVAL, "dx overlaps x");
  return norm_bwd_impl(dy, lddy, x, ldx, stats, n_rows, max_rows, gamma, past, ldp, d, dx, lddx, dgamma, dbeta, ws, stream);
}

size_t mtgnn_softmax_loss_save_bytes(const mtgnn_loss_dims* d, int64_t max_rows) {
  if (check_loss(d) != MTGNN_OK || check_rows(max_rows, 1) != MTGNN_OK) return 0;
  return loss_save(d, max_rows);
}

size_t mtgnn_softmax_loss_ws_bytes(const mtgnn_loss_dims* d, int64_t max_rows, int32_t backward) {
  if (check_loss(d) != MTGNN_OK || check_rows(max_rows, 1) != MTGNN_OK) return 0;
  const size_t fwd = loss_ws(d, max_rows, false);
  return backward ? std::max(fwd, loss_ws(d, max_rows, true)) : fwd;
}

mtgnn_status mtgnn_softmax_loss(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const void* W,
                                const float* b, const int32_t* label, const mtgnn_loss_dims* d, float* loss,
                                float* row_loss, void* save, void* ws, size_t ws_bytes, hipStream_t stream) {
  MTGNN_TRY(check_loss(d));
  MTGNN_TRY(check_rows(max_rows, 1));
  if (max_rows == 0) return fail(MTGNN_EINVAL, "max_rows == 0 (no row: the loss is zero; skip the call)");
  REQ(x, "x");
  REQ(W, "W");
  REQ(label, "label");
  REQ(loss, "loss");
  REQ(ws, "ws");
  STRIDE(ldx, d->d, "ldx");
  if (!loss_fits(d, max_rows)) return fail(MTGNN_EUNSUPPORTED, "max_rows times n, or n times d");
  if (ws_bytes < loss_ws(d, max_rows, false)) return fail(MTGNN_EWORKSPACE, "softmax_loss ws");
  MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  MTGNN_TRY(check_aligned(save, "save is not 16-byte aligned"));
  return loss_impl(x, ldx, n_rows, max_rows, W, b, label, d, loss, row_loss, save, ws, stream);
}

mtgnn_status mtgnn_softmax_loss_bwd(const int32_t* n_rows, int64_t max_rows, const void* W, const float* b,
                                    const int32_t* label, const mtgnn_loss_dims* d, const void* save, const float* dloss,
                                    float* dx, int64_t lddx, float* dW, float* db, void* ws, size_t ws_bytes,
                                    hipStream_t stream) {
  MTGNN_TRY(check_loss(d));
  MTGNN_TRY(check_rows(max_rows, 1));
  if (max_rows == 0) return fail(MTGNN_EINVAL, "max_rows == 0 (no row: every gradient is zero; skip the call)");
  if (!dx && !dW && !db) return MTGNN_OK;
  REQ(W, "W");
  REQ(label, "label");
  REQ(save, "save");
  REQ(ws, "ws");
  if (dx) STRIDE(lddx, d->d, "lddx");
  if (!loss_fits(d, max_rows)) return fail(MTGNN_EUNSUPPORTED, "max_rows times n, or n times d");
  if (ws_bytes < loss_ws(d, max_rows, true)) return fail(MTGNN_EWORKSPACE, "softmax_loss_bwd ws");
  MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  MTGNN_TRY(check_aligned(save, "save is not 16-byte aligned"));
  const int64_t nd = (int64_t)d->n * d->d, to = ((max_rows - 1) * lddx + d->d) * 4;
  if (overlap(Rows{dx, to, to}, Rows{W, nd * bytes_of(d->dtype), nd * bytes_of(d->dtype)}, 1)) return fail(MTGNN_EINVAL, "dx overlaps W");
  if (overlap(Rows{dx, to, to}, Rows{dW, nd * 4, nd * 4}, 1)) return fail(MTGNN_EINVAL, "dx overlaps dW");
  if (overlap(Rows{dW, nd * 4, nd * 4}, Rows{W, nd * bytes_of(d->dtype), nd * bytes_of(d->dtype)}, 1))
    return fail(MTGNN_EINVAL, "dW overlaps W");
  return loss_bwd_impl(n_rows, max_rows, W, b, label, d, save, dloss, dx, lddx, dW, db, ws, stream);
}

mtgnn_status mtgnn_adamw_step(const mtgnn_adamw_tensor* tensors, int64_t n, const mtgnn_adam_config* cfg,
                              const int32_t* step, hipStream_t stream) {
  if (n < 0) return fail(MTGNN_EINVAL, "n");
  REQ(cfg, "cfg");
  if (!(cfg->beta1 >= 0 && cfg->beta1 < 1) || !(cfg->beta2 >= 0 && cfg->beta2 < 1)) return fail(MTGNN_EINVAL, "beta1 or beta2 not in [0, 1)");
  if (!(cfg->eps >= 0) || !std::isfinite(cfg->eps)) return fail(MTGNN_EINVAL, "eps is negative or not finite");
  if (!std::isfinite(cfg->lr)) return fail(MTGNN_EINVAL, "lr is not finite");
  if (!step && cfg->t < 1) return fail(MTGNN_EINVAL, "t < 1");
  if (n > 0) REQ(tensors, "tensors");
  for (int64_t i = 0; i < n; ++i) {
    const mtgnn_adamw_tensor& t = tensors[i];
    if (t.n < 0) return fail(MTGNN_EINVAL, "a tensor's n");
    if (t.n > int64_t(1) << 33) return fail(MTGNN_EUNSUPPORTED, "a tensor's n > 2^33");
    if (!std::isfinite(t.decay)) return fail(MTGNN_EINVAL, "a tensor's decay is not finite");
    if ((t.m_exp == nullptr) != (t.v_exp == nullptr)) return fail(MTGNN_EINVAL, "one of m_exp and v_exp is NULL");
    if (t.n == 0) continue;
    REQ(t.param, "param");
    REQ(t.grad, "grad");
    REQ(t.m, "m");
    REQ(t.v, "v");
  }
  return adamw_impl(tensors, n, cfg, step, stream);
}

}  // extern "C"
