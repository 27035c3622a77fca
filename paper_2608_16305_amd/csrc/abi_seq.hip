// C ABI of the state-space layer's operators: argument validation (host only, before any HIP call) and dispatch.
#include <algorithm>

#include "ops.h"

using namespace mtgnn;

#define REQ(p, name) \
  if (!(p)) return fail(MTGNN_EINVAL, name " is NULL")

namespace {

constexpr int64_t MAX_ROWS = (int64_t(1) << 31) - 64;   // a tile past the last row is still an int32
constexpr int MAX_WIDTH = 1 << 20;   // channels, columns

bool dtype_ok(int t) { return t == MTGNN_F32 || t == MTGNN_BF16; }

mtgnn_status check_rows(int64_t rows, int64_t width) {
  if (rows < 0 || rows >= MAX_ROWS) return fail(MTGNN_EINVAL, "max_rows");
  if (rows * width >= MAX_ROWS * 256) return fail(MTGNN_EUNSUPPORTED, "max_rows times width");   // grid of one launch
  return MTGNN_OK;
}

mtgnn_status check_seqs(const mtgnn_seqs* q, int64_t width) {
  if (!q) return fail(MTGNN_EINVAL, "seqs is NULL");
  MTGNN_TRY(check_rows(q->max_rows, width));
  if (q->max_seq < 0 || q->max_seq > (int64_t(1) << 30)) return fail(MTGNN_EINVAL, "max_seq");
  if (q->max_seq * width >= MAX_ROWS * 256) return fail(MTGNN_EUNSUPPORTED, "max_seq times width");
  if (q->n_slots < 0 || q->n_slots >= MAX_ROWS) return fail(MTGNN_EINVAL, "n_slots");
  if (q->max_seq > 0 && q->max_rows > 0) REQ(q->off, "off");
  return MTGNN_OK;
}
// A launch with a thread to each of rows x width (work items are a 32-bit number).
mtgnn_status check_items(int64_t rows, int64_t width, const char* what) {
  return rows * width > (int64_t(1) << 32) - 256 ? fail(MTGNN_EUNSUPPORTED, what) : MTGNN_OK;
}
mtgnn_status check_aligned(const void* p, const char* what) {   // (read by whole words, by the scalar unit too)
  return (uintptr_t)p % 16 ? fail(MTGNN_EINVAL, what) : MTGNN_OK;
}
// A matrix of rows in memory, in bytes.
struct Rows {
  const void* p;
  int64_t ld, width;
};
// Whether two of `rows` rows share a byte.  Exact where their rows are as far apart (column ranges of one matrix may lie side
// by side); else whether the memory from the first row to the last does.
bool overlap(const Rows& a, const Rows& b, int64_t rows) {
  const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  if (!a.p || !b.p || d >= (rows - 1) * a.ld + a.width || -d >= (rows - 1) * b.ld + b.width) return false;
  if (a.ld != b.ld) return true;
  const int64_t c = (d % a.ld + a.ld) % a.ld;   // b's first column, seen from a's
  return c < a.width || c + b.width > a.ld;
}
int64_t bytes_of(int dtype) { return dtype == MTGNN_BF16 ? 2 : 4; }
bool no_rows(const mtgnn_seqs* q) { return q->max_rows == 0 || q->max_seq == 0; }

#define STRIDE(ld, width, name) \
  if ((ld) < (width)) return fail(MTGNN_EINVAL, name " is less than the row's width")

mtgnn_status check_linear(const mtgnn_linear_dims* d) {
  if (!d) return fail(MTGNN_EINVAL, "dims is NULL");
  if (!dtype_ok(d->dtype)) return fail(MTGNN_EUNSUPPORTED, "dtype");
  if (d->act < MTGNN_ACT_NONE || d->act > MTGNN_ACT_GELU) return fail(MTGNN_EUNSUPPORTED, "act");
  if (d->d_in <= 0 || d->d_out <= 0) return fail(MTGNN_EINVAL, "non-positive dimension");
  if (d->d_in > MAX_WIDTH || d->d_out > MAX_WIDTH) return fail(MTGNN_EUNSUPPORTED, "width > 2^20");
  return MTGNN_OK;
}

mtgnn_status check_conv(const mtgnn_conv_dims* d) {
  if (!d) return fail(MTGNN_EINVAL, "dims is NULL");
  if (!dtype_ok(d->dtype)) return fail(MTGNN_EUNSUPPORTED, "dtype");
  if (d->act != MTGNN_ACT_NONE && d->act != MTGNN_ACT_SILU) return fail(MTGNN_EUNSUPPORTED, "act");
  if (d->d <= 0) return fail(MTGNN_EINVAL, "non-positive dimension");
  if (d->d > MAX_WIDTH) return fail(MTGNN_EUNSUPPORTED, "d > 2^20");
  if (d->width < 2 || d->width > 4) return fail(MTGNN_EUNSUPPORTED, "width is not 2, 3 or 4");
  return MTGNN_OK;
}

mtgnn_status check_scan(const mtgnn_scan_dims* d) {
  if (!d) return fail(MTGNN_EINVAL, "dims is NULL");
  if (!dtype_ok(d->dtype)) return fail(MTGNN_EUNSUPPORTED, "dtype");
  if (d->d <= 0 || d->n <= 0 || d->groups <= 0) return fail(MTGNN_EINVAL, "non-positive dimension");
  if (d->d % d->groups != 0) return fail(MTGNN_EINVAL, "groups does not divide d");
  if (d->d > MAX_WIDTH) return fail(MTGNN_EUNSUPPORTED, "d > 2^20");
  if (d->n > 64) return fail(MTGNN_EUNSUPPORTED, "n > 64");
  return MTGNN_OK;
}

mtgnn_status check_inputs(const mtgnn_scan_inputs* in, const mtgnn_scan_dims* d) {
  REQ(in, "in");
  REQ(in->x, "x");
  REQ(in->delta, "delta");
  REQ(in->B, "B");
  REQ(in->C, "C");
  REQ(in->A, "A");
  STRIDE(in->ldx, d->d, "ldx");
  STRIDE(in->lddelta, d->d, "lddelta");
  STRIDE(in->ldB, (int64_t)d->groups * d->n, "ldB");
  STRIDE(in->ldC, (int64_t)d->groups * d->n, "ldC");
  if (in->z) STRIDE(in->ldz, d->d, "ldz");
  return MTGNN_OK;
}

}  // namespace

extern "C" {

size_t mtgnn_linear_ws_bytes(const mtgnn_linear_dims* d, int64_t max_rows, int32_t backward) {
  if (check_linear(d) != MTGNN_OK || check_rows(max_rows, d->d_out) != MTGNN_OK) return 0;
  const size_t fwd = linear_ws(d, max_rows, false);
  return backward ? std::max(fwd, linear_ws(d, max_rows, true)) : fwd;
}

mtgnn_status mtgnn_linear(const void* x, int64_t ldx, const int32_t* n_rows, int64_t max_rows, const void* W,
                          const float* b, const void* residual, int64_t ldr, const mtgnn_linear_dims* d, void* y,
                          int64_t ldy, float* pre, void* ws, size_t ws_bytes, hipStream_t stream) {
  MTGNN_TRY(check_linear(d));
  MTGNN_TRY(check_rows(max_rows, d->d_out));
  if (max_rows == 0) return MTGNN_OK;
  REQ(x, "x");
  REQ(W, "W");
  REQ(y, "y");
  STRIDE(ldx, d->d_in, "ldx");
  STRIDE(ldy, d->d_out, "ldy");
  if (residual) STRIDE(ldr, d->d_out, "ldr");
  if (!linear_fits(d, max_rows, false)) return fail(MTGNN_EUNSUPPORTED, "max_rows times width");
  const size_t need = linear_ws(d, max_rows, false);
  if (ws_bytes < need) return fail(MTGNN_EWORKSPACE, "linear ws");
  if (need) REQ(ws, "ws");
  MTGNN_TRY(check_aligned(need ? ws : nullptr, "ws is not 16-byte aligned"));
  return linear_impl(x, ldx, n_rows, max_rows, W, b, residual, ldr, d, y, ldy, pre, ws, ws_bytes, stream);
}

mtgnn_status mtgnn_linear_bwd(const float* dy, int64_t lddy, const float* pre, const void* x, int64_t ldx,
                              const int32_t* n_rows, int64_t max_rows, const void* W, const mtgnn_linear_dims* d,
                              float* dx, int64_t lddx, float* dW, float* db, void* ws, size_t ws_bytes,
                              hipStream_t stream) {
  MTGNN_TRY(check_linear(d));
  MTGNN_TRY(check_rows(max_rows, d->d_out));
  REQ(dW, "dW");
  if (max_rows == 0) return fail(MTGNN_EINVAL, "max_rows == 0 (no row: every gradient is zero; skip the call)");
  REQ(dy, "dy");
  REQ(x, "x");
  REQ(W, "W");
  if (d->act != MTGNN_ACT_NONE) REQ(pre, "pre");
  STRIDE(lddy, d->d_out, "lddy");
  STRIDE(ldx, d->d_in, "ldx");
  if (dx) STRIDE(lddx, d->d_in, "lddx");
  if (!linear_fits(d, max_rows, true)) return fail(MTGNN_EUNSUPPORTED, "max_rows times width");
  const size_t need = linear_ws(d, max_rows, true);
  if (ws_bytes < need) return fail(MTGNN_EWORKSPACE, "linear_bwd ws");
  if (need) REQ(ws, "ws");
  MTGNN_TRY(check_aligned(need ? ws : nullptr, "ws is not 16-byte aligned"));
  // dW is made from x, and from dy where that is the slope, after dx is written
  const int64_t e = bytes_of(d->dtype);
  const Rows to{dx, lddx * 4, (int64_t)d->d_in * 4};
  if (overlap(to, Rows{x, ldx * e, d->d_in * e}, max_rows)) return fail(MTGNN_EINVAL, "dx overlaps x");
  if (d->act == MTGNN_ACT_NONE && overlap(to, Rows{dy, lddy * 4, (int64_t)d->d_out * 4}, max_rows))
    return fail(MTGNN_EINVAL, "dx overlaps dy (without an activation)");
  return linear_bwd_impl(dy, lddy, pre, x, ldx, n_rows, max_rows, W, d, dx, lddx, dW, db, ws, ws_bytes, stream);
}

size_t mtgnn_causal_conv_save_bytes(const mtgnn_conv_dims* d, int64_t max_seq) {
  if (check_conv(d) != MTGNN_OK || max_seq < 0 || max_seq > (int64_t(1) << 30)) return 0;
  return conv_save(d, max_seq);
}

size_t mtgnn_causal_conv_ws_bytes(const mtgnn_conv_dims* d, int64_t max_rows) {
  if (check_conv(d) != MTGNN_OK || check_rows(max_rows, d->d) != MTGNN_OK) return 0;
  return conv_ws(d, max_rows);
}

mtgnn_status mtgnn_causal_conv(const mtgnn_seqs* q, const void* x, int64_t ldx, const void* w, const float* b,
                               const mtgnn_conv_dims* d, const void* state_in, void* state_out, void* y,
                               int64_t ldy, void* save, hipStream_t stream) {
  MTGNN_TRY(check_conv(d));
  MTGNN_TRY(check_seqs(q, d->d));
  if (no_rows(q)) return MTGNN_OK;
  REQ(x, "x");
  REQ(w, "w");
  REQ(y, "y");
  STRIDE(ldx, d->d, "ldx");
  STRIDE(ldy, d->d, "ldy");
  if (state_out || save) MTGNN_TRY(check_items(q->max_seq, d->d, "max_seq times d >= 2^32"));
  return conv_impl(q, x, ldx, w, b, d, state_in, state_out, y, ldy, save, stream);
}

mtgnn_status mtgnn_causal_conv_bwd(const mtgnn_seqs* q, const float* dy, int64_t lddy, const void* x, int64_t ldx,
                                   const void* w, const float* b, const mtgnn_conv_dims* d, const void* save,
                                   float* dx, int64_t lddx, float* dw, float* db, void* ws, size_t ws_bytes,
                                   hipStream_t stream) {
  MTGNN_TRY(check_conv(d));
  MTGNN_TRY(check_seqs(q, d->d));
  REQ(dw, "dw");
  if (no_rows(q)) return fail(MTGNN_EINVAL, "no rows (every gradient is zero; skip the call)");
  REQ(dy, "dy");
  REQ(x, "x");
  REQ(w, "w");
  REQ(dx, "dx");
  STRIDE(lddy, d->d, "lddy");
  STRIDE(ldx, d->d, "ldx");
  STRIDE(lddx, d->d, "lddx");
  if (ws_bytes < conv_ws(d, q->max_rows)) return fail(MTGNN_EWORKSPACE, "causal_conv_bwd ws");
  REQ(ws, "ws");
  MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  // a chunk reads rows of its neighbours, which may have written their dx by then
  const int64_t e = bytes_of(d->dtype), w4 = (int64_t)d->d * 4;
  const Rows to{dx, lddx * 4, w4};
  if (overlap(to, Rows{dy, lddy * 4, w4}, q->max_rows)) return fail(MTGNN_EINVAL, "dx overlaps dy");
  if (overlap(to, Rows{x, ldx * e, d->d * e}, q->max_rows)) return fail(MTGNN_EINVAL, "dx overlaps x");
  return conv_bwd_impl(q, dy, lddy, x, ldx, w, b, d, save, dx, lddx, dw, db, ws, stream);
}

mtgnn_status mtgnn_causal_conv_step(const int32_t* slot, const int32_t* n_rows, int64_t max_rows, int64_t n_slots,
                                    const void* x, int64_t ldx, const void* w, const float* b,
                                    const mtgnn_conv_dims* d, const void* state_in, void* state_out, void* y,
                                    int64_t ldy, hipStream_t stream) {
  MTGNN_TRY(check_conv(d));
  MTGNN_TRY(check_rows(max_rows, d->d));
  if (n_slots < 0 || n_slots >= MAX_ROWS) return fail(MTGNN_EINVAL, "n_slots");
  if (max_rows == 0) return MTGNN_OK;
  REQ(x, "x");
  REQ(w, "w");
  REQ(y, "y");
  STRIDE(ldx, d->d, "ldx");
  STRIDE(ldy, d->d, "ldy");
  MTGNN_TRY(check_items(max_rows, d->d, "max_rows times d >= 2^32"));
  return conv_step_impl(slot, n_rows, max_rows, n_slots, x, ldx, w, b, d, state_in, state_out, y, ldy, stream);
}

size_t mtgnn_selective_scan_ws_bytes(const mtgnn_scan_dims* d, int64_t max_rows, int64_t max_seq, int32_t backward) {
  if (check_scan(d) != MTGNN_OK || check_rows(max_rows, d->d) != MTGNN_OK || max_seq < 0) return 0;
  const size_t fwd = scan_ws(d, max_rows, false);
  return backward ? std::max(fwd, scan_ws(d, max_rows, true)) : fwd;
}

size_t mtgnn_selective_scan_save_bytes(const mtgnn_scan_dims* d, int64_t max_rows, int64_t max_seq, int32_t carried) {
  if (check_scan(d) != MTGNN_OK || check_rows(max_rows, d->d) != MTGNN_OK || max_seq < 0 ||
      max_seq > (int64_t(1) << 30))
    return 0;
  return scan_save(d, max_rows, max_seq, carried != 0);
}

mtgnn_status mtgnn_selective_scan(const mtgnn_seqs* q, const mtgnn_scan_inputs* in, const mtgnn_scan_dims* d,
                                  const float* state_in, float* state_out, void* y, int64_t ldy, void* save, void* ws,
                                  size_t ws_bytes, hipStream_t stream) {
  MTGNN_TRY(check_scan(d));
  MTGNN_TRY(check_seqs(q, d->d));
  if (no_rows(q)) return MTGNN_OK;
  MTGNN_TRY(check_inputs(in, d));
  REQ(y, "y");
  STRIDE(ldy, d->d, "ldy");
  if (ws_bytes < scan_ws(d, q->max_rows, false)) return fail(MTGNN_EWORKSPACE, "selective_scan ws");
  REQ(ws, "ws");
  MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  MTGNN_TRY(check_aligned(save, "save is not 16-byte aligned"));
  return scan_impl(q, in, d, state_in, state_out, y, ldy, save, ws, stream);
}

mtgnn_status mtgnn_selective_scan_bwd(const mtgnn_seqs* q, const float* dy, int64_t lddy, const mtgnn_scan_inputs* in,
                                      const mtgnn_scan_dims* d, const void* save, const mtgnn_scan_grads* g, void* ws,
                                      size_t ws_bytes, hipStream_t stream) {
  MTGNN_TRY(check_scan(d));
  MTGNN_TRY(check_seqs(q, d->d));
  REQ(g, "grads");
  if (no_rows(q)) return fail(MTGNN_EINVAL, "no rows (every gradient is zero; skip the call)");
  MTGNN_TRY(check_inputs(in, d));
  REQ(dy, "dy");
  REQ(save, "save");
  REQ(g->dx, "dx");
  REQ(g->ddelta, "ddelta");
  REQ(g->dB, "dB");
  REQ(g->dC, "dC");
  REQ(g->dA, "dA");
  if ((g->dz != nullptr) != (in->z != nullptr)) return fail(MTGNN_EINVAL, "dz must be given iff z is");
  if ((g->dD != nullptr) != (in->D != nullptr)) return fail(MTGNN_EINVAL, "dD must be given iff D is");
  if ((g->ddelta_bias != nullptr) != (in->delta_bias != nullptr))
    return fail(MTGNN_EINVAL, "ddelta_bias must be given iff delta_bias is");
  STRIDE(lddy, d->d, "lddy");
  STRIDE(g->lddx, d->d, "lddx");
  STRIDE(g->ldddelta, d->d, "ldddelta");
  STRIDE(g->lddB, (int64_t)d->groups * d->n, "lddB");
  STRIDE(g->lddC, (int64_t)d->groups * d->n, "lddC");
  if (g->dz) STRIDE(g->lddz, d->d, "lddz");
  MTGNN_TRY(check_items(q->max_rows, 2 * (int64_t)d->groups * d->n, "max_rows times 2 groups n >= 2^32"));
  if (ws_bytes < scan_ws(d, q->max_rows, true)) return fail(MTGNN_EWORKSPACE, "selective_scan_bwd ws");
  REQ(ws, "ws");
  MTGNN_TRY(check_aligned(ws, "ws is not 16-byte aligned"));
  MTGNN_TRY(check_aligned(save, "save is not 16-byte aligned"));
  return scan_bwd_impl(q, dy, lddy, in, d, save, g, ws, stream);
}

mtgnn_status mtgnn_selective_scan_step(const int32_t* slot, const int32_t* n_rows, int64_t max_rows, int64_t n_slots,
                                       const mtgnn_scan_inputs* in, const mtgnn_scan_dims* d, const float* state_in,
                                       float* state_out, void* y, int64_t ldy, hipStream_t stream) {
  MTGNN_TRY(check_scan(d));
  MTGNN_TRY(check_rows(max_rows, d->d));
  if (n_slots < 0 || n_slots >= MAX_ROWS) return fail(MTGNN_EINVAL, "n_slots");
  if (max_rows == 0) return MTGNN_OK;
  MTGNN_TRY(check_inputs(in, d));
  REQ(y, "y");
  STRIDE(ldy, d->d, "ldy");
  MTGNN_TRY(check_items(max_rows, d->d, "max_rows times d >= 2^32"));
  return scan_step_impl(slot, n_rows, max_rows, n_slots, in, d, state_in, state_out, y, ldy, stream);
}

}  // extern "C"
