// Checks that the entry points of the layer and model operators share (host only, before any HIP call).
#pragma once

#include "ops.h"

#define REQ(p, name) \
  if (!(p)) return fail(MTGNN_EINVAL, name " is NULL")
#define STRIDE(ld, width, name) \
  if ((ld) < (width)) return fail(MTGNN_EINVAL, name " is less than the row's width")

namespace mtgnn {

namespace {

constexpr int64_t MAX_ROWS = (int64_t(1) << 31) - 64;   // a tile past the last row is still an int32
constexpr int MAX_WIDTH = 1 << 20;   // channels, columns

inline bool dtype_ok(int t) { return t == MTGNN_F32 || t == MTGNN_BF16; }

inline mtgnn_status check_rows(int64_t rows, int64_t width) {
  if (rows < 0 || rows >= MAX_ROWS) return fail(MTGNN_EINVAL, "max_rows");
  if (rows * width >= MAX_ROWS * 256) return fail(MTGNN_EUNSUPPORTED, "max_rows times width");   // grid of one launch
  return MTGNN_OK;
}
// A launch with a thread to each of rows x width (work items are a 32-bit number).
inline mtgnn_status check_items(int64_t rows, int64_t width, const char* what) {
  return rows * width > (int64_t(1) << 32) - 256 ? fail(MTGNN_EUNSUPPORTED, what) : MTGNN_OK;
}
inline mtgnn_status check_aligned(const void* p, const char* what) {   // (read by whole words, by the scalar unit too)
  return (uintptr_t)p % 16 ? fail(MTGNN_EINVAL, what) : MTGNN_OK;
}
// A matrix of rows in memory, in bytes.
struct Rows {
  const void* p;
  int64_t ld, width;
};
// Whether two of `rows` rows share a byte.  Exact where their rows are as far apart (column ranges of one matrix may lie side
// by side); else whether the memory from the first row to the last does.
inline bool overlap(const Rows& a, const Rows& b, int64_t rows) {
  const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  if (!a.p || !b.p || d >= (rows - 1) * a.ld + a.width || -d >= (rows - 1) * b.ld + b.width) return false;
  if (a.ld != b.ld) return true;
  const int64_t c = (d % a.ld + a.ld) % a.ld;   // b's first column, seen from a's
  return c < a.width || c + b.width > a.ld;
}
inline int64_t bytes_of(int dtype) { return dtype == MTGNN_BF16 ? 2 : 4; }

}  // namespace

}  // namespace mtgnn
