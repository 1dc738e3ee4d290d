// C ABI of the word-model operators (include/lda_ops.h): argument checks and
// error reporting around the launchers of ops_norm.hip and ops_product.hip.
#include <cmath>
#include <string>

#include "handle.h"
#include "ops_internal.h"

using namespace lda;
using namespace lda::ops;

namespace {

// The message of lda_last_error(NULL); a message that finds no host memory is
// left out, the status stands.
lda_status refuse(lda_status st, const char *msg) noexcept {
  try {
    g_create_error = msg;
  } catch (...) {
    g_create_error.clear();
  }
  return st;
}

lda_status launched(hipError_t e) noexcept {
  if (e == hipSuccess) return LDA_OK;
  return refuse(e == hipErrorOutOfMemory ? LDA_E_NOMEM : LDA_E_DEVICE, hipGetErrorString(e));
}

#define REQUIRE(cond, st, msg)               \
  do {                                       \
    if (!(cond)) return refuse((st), (msg)); \
  } while (0)

// A matrix argument of `rows` rows and `cols` columns (an output also needs
// room between its rows); no pointer is needed where there are no rows.
lda_status check_in(const void *p, int64_t ld, int64_t rows, const char *msg) {
  REQUIRE(p || rows == 0, LDA_E_ARG, msg);
  REQUIRE(ld >= 0, LDA_E_ARG, "a row stride must not be negative");
  return LDA_OK;
}

lda_status check_out(const void *p, int64_t ld, int64_t rows, int64_t cols, const char *msg) {
  REQUIRE(p || rows == 0, LDA_E_ARG, msg);
  REQUIRE(ld >= cols || rows <= 1, LDA_E_ARG, "an output's row stride must be at least its columns");
  return LDA_OK;
}

lda_status check_rows(int dtype, int64_t rows) {
  REQUIRE(dtype >= LDA_F32 && dtype <= LDA_F16, LDA_E_ARG, "unknown element type");
  REQUIRE(rows >= 0, LDA_E_ARG, "rows must not be negative");
  REQUIRE(rows <= LDA_OPS_MAX_ROWS, LDA_E_RANGE, "more rows than LDA_OPS_MAX_ROWS");
  return LDA_OK;
}

lda_status check_cols(int64_t cols) {
  REQUIRE(cols >= 1, LDA_E_ARG, "widths must be positive");
  REQUIRE(cols <= LDA_OPS_MAX_COLS, LDA_E_RANGE, "a width is more than LDA_OPS_MAX_COLS");
  return LDA_OK;
}

// Of a product's result: its tiles (the smallest are 64 x 64, four times as many)
// are counted in 32 bits.
lda_status check_product(int64_t rows, int64_t cols) {
  REQUIRE(ceil_div(rows, 128) * ceil_div(cols, 128) <= LDA_OPS_MAX_TILES, LDA_E_RANGE,
          "a product has more than LDA_OPS_MAX_TILES tiles of 128 x 128");
  return LDA_OK;
}

lda_status check_norm(const lda_norm_args *a, bool backward) {
  REQUIRE(a, LDA_E_ARG, "args is NULL");
  LDA_TRY(check_rows(a->dtype, a->rows));
  LDA_TRY(check_cols(a->cols));
  LDA_TRY(check_in(a->x, a->ldx, a->rows, "x is NULL"));
  REQUIRE((a->mean && a->rstd) || a->rows == 0, LDA_E_ARG, "mean or rstd is NULL");
  if (!backward) {
    REQUIRE(std::isfinite(a->eps) && a->eps >= 0.0f, LDA_E_ARG, "eps must be finite and not negative");
    REQUIRE((a->weight == nullptr) == (a->bias == nullptr), LDA_E_ARG, "weight and bias must be given together");
    return check_out(a->y, a->ldy, a->rows, a->cols, "y is NULL");
  }
  REQUIRE((a->dweight == nullptr) == (a->dbias == nullptr), LDA_E_ARG, "dweight and dbias must be given together");
  LDA_TRY(check_in(a->dy, a->lddy, a->rows, "dy is NULL"));
  return check_out(a->dx, a->lddx, a->rows, a->cols, "dx is NULL");
}

lda_status check_gated(const lda_gated_args *a, bool backward) {
  REQUIRE(a, LDA_E_ARG, "args is NULL");
  LDA_TRY(check_rows(a->dtype, a->rows));
  REQUIRE(a->act >= LDA_SILU && a->act <= LDA_SIGMOID, LDA_E_ARG, "unknown activation");
  LDA_TRY(check_cols(a->width));
  LDA_TRY(check_cols(a->hidden));
  LDA_TRY(check_product(a->rows, 2 * round_up(a->hidden, 64)));
  LDA_TRY(check_product(2 * round_up(a->hidden, 64), a->width));
  LDA_TRY(check_product(a->rows, a->width));
  LDA_TRY(check_in(a->x, a->ldx, a->rows, "x is NULL"));
  LDA_TRY(check_in(a->w_gate, a->ld_gate, 1, "w_gate is NULL"));
  LDA_TRY(check_in(a->w_value, a->ld_value, 1, "w_value is NULL"));
  if (!backward) return check_out(a->h, a->ldh, a->rows, a->hidden, "h is NULL");
  LDA_TRY(check_in(a->dh, a->lddh, a->rows, "dh is NULL"));
  REQUIRE(a->dw_gate && a->dw_value, LDA_E_ARG, "dw_gate or dw_value is NULL");
  return check_out(a->dx, a->lddx, a->rows, a->width, "dx is NULL");
}

lda_status check_xent(const lda_xent_args *a, bool backward) {
  REQUIRE(a, LDA_E_ARG, "args is NULL");
  LDA_TRY(check_rows(a->dtype, a->rows));
  LDA_TRY(check_cols(a->width));
  REQUIRE(a->vocab >= 1, LDA_E_ARG, "vocab must be positive");
  REQUIRE(a->vocab <= LDA_OPS_MAX_VOCAB, LDA_E_RANGE, "more words than LDA_OPS_MAX_VOCAB");
  LDA_TRY(check_product(a->rows, a->vocab));
  LDA_TRY(check_product(a->vocab, a->width));
  LDA_TRY(check_product(a->rows, a->width));
  LDA_TRY(check_in(a->x, a->ldx, a->rows, "x is NULL"));
  LDA_TRY(check_in(a->weight, a->ld_weight, 1, "weight is NULL"));
  REQUIRE(a->labels || a->rows == 0, LDA_E_ARG, "labels is NULL");
  REQUIRE(a->lse || a->rows == 0, LDA_E_ARG, "lse is NULL");
  if (!backward) {
    REQUIRE(a->loss || a->rows == 0, LDA_E_ARG, "loss is NULL");
    return LDA_OK;
  }
  REQUIRE(a->dloss || a->rows == 0, LDA_E_ARG, "dloss is NULL");
  REQUIRE(a->dweight, LDA_E_ARG, "dweight is NULL");
  REQUIRE((a->bias == nullptr) == (a->dbias == nullptr), LDA_E_ARG, "dbias must be given if and only if bias is");
  return check_out(a->dx, a->lddx, a->rows, a->width, "dx is NULL");
}

// Counts the workspace of `fn` for `a`, and with `bytes` NULL runs it in the
// caller's.
template <typename Args, typename Fn>
lda_status with_workspace(const Args *a, Fn fn, size_t *bytes) {
  Arena count;
  LDA_TRY(launched(fn(*a, count, true)));
  if (bytes) {
    *bytes = count.used;
    return LDA_OK;
  }
  REQUIRE(a->workspace_bytes >= count.used && (a->workspace || !count.used), LDA_E_ARG, "the workspace is too small");
  REQUIRE(reinterpret_cast<uintptr_t>(a->workspace) % 256 == 0, LDA_E_ARG, "the workspace must be 256-byte aligned");
  Arena ws;
  ws.base = static_cast<char *>(a->workspace);
  return launched(fn(*a, ws, false));
}

}  // namespace

extern "C" {

lda_status lda_layer_norm(const lda_norm_args *a) {
  LDA_TRY(check_norm(a, false));
  return launched(norm_forward(*a));
}

lda_status lda_layer_norm_backward_workspace(const lda_norm_args *a, size_t *bytes) {
  REQUIRE(bytes, LDA_E_ARG, "bytes is NULL");
  LDA_TRY(check_norm(a, true));
  return with_workspace(a, norm_backward, bytes);
}

lda_status lda_layer_norm_backward(const lda_norm_args *a) {
  LDA_TRY(check_norm(a, true));
  return with_workspace(a, norm_backward, nullptr);
}

lda_status lda_gated_workspace(const lda_gated_args *a, size_t *bytes) {
  REQUIRE(bytes, LDA_E_ARG, "bytes is NULL");
  LDA_TRY(check_gated(a, false));
  return with_workspace(a, gated_forward, bytes);
}

lda_status lda_gated(const lda_gated_args *a) {
  LDA_TRY(check_gated(a, false));
  return with_workspace(a, gated_forward, nullptr);
}

lda_status lda_gated_backward_workspace(const lda_gated_args *a, size_t *bytes) {
  REQUIRE(bytes, LDA_E_ARG, "bytes is NULL");
  LDA_TRY(check_gated(a, true));
  return with_workspace(a, gated_backward, bytes);
}

lda_status lda_gated_backward(const lda_gated_args *a) {
  LDA_TRY(check_gated(a, true));
  return with_workspace(a, gated_backward, nullptr);
}

lda_status lda_softmax_xent_workspace(const lda_xent_args *a, size_t *bytes) {
  REQUIRE(bytes, LDA_E_ARG, "bytes is NULL");
  LDA_TRY(check_xent(a, false));
  return with_workspace(a, xent_forward, bytes);
}

lda_status lda_softmax_xent(const lda_xent_args *a) {
  LDA_TRY(check_xent(a, false));
  return with_workspace(a, xent_forward, nullptr);
}

lda_status lda_softmax_xent_backward_workspace(const lda_xent_args *a, size_t *bytes) {
  REQUIRE(bytes, LDA_E_ARG, "bytes is NULL");
  LDA_TRY(check_xent(a, true));
  return with_workspace(a, xent_backward, bytes);
}

lda_status lda_softmax_xent_backward(const lda_xent_args *a) {
  LDA_TRY(check_xent(a, true));
  return with_workspace(a, xent_backward, nullptr);
}

}  // extern "C"
