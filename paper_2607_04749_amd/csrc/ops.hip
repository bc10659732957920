// ops.hip -- the C ABI of the operators of a training step (include/etc.h):
// argument checks and dispatch.  Nothing here allocates or throws.
#include <hip/hip_runtime.h>

#include <cmath>

#include "etc.h"
#include "ops.hpp"
#include "ops_check.hpp"

namespace {

int check_drop(const etc_dropout_desc& d, int64_t rows, etc::Drop* out) {
  if (!(d.p >= 0.0 && d.p <= 1.0)) return fail(ETC_ERR_INVALID_ARG, "dropout: p must lie in 0 .. 1");
  if (d.reserved != 0) return fail(ETC_ERR_INVALID_ARG, "dropout: reserved must be 0");
  if (d.row0 < 0 || d.row0 > INT64_MAX - rows) return fail(ETC_ERR_INVALID_ARG, "dropout: row0 is out of range");
  out->k0 = uint32_t(d.seed);
  out->k1 = uint32_t(d.seed >> 32);
  out->call = d.call;
  out->limit = uint32_t(std::floor(65536.0 * d.p + 0.5));
  out->row0 = uint64_t(d.row0);
  out->scale = out->limit < 65536 ? float(65536.0 / (65536 - out->limit)) : 0.0f;
  return ETC_OK;
}

// the ids row0 .. row0 + rows of a table: an id minus row0 must not wrap into them
int check_row0(int64_t row0, int64_t rows) {
  return row0 <= INT64_MAX - rows ? int(ETC_OK) : fail(ETC_ERR_INVALID_ARG, "row0 is out of range");
}

}  // namespace

extern "C" {

int etc_embed(const etc_embed_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  etc::Drop drop;
  int rc;
  if ((rc = check_ids(a->tokens, "tokens")) || (rc = check_matrix(a->table, "table", kIn)) ||
      (rc = check_matrix(a->out, "out", kOut)) || (rc = check_scale(a->scale)) ||
      (rc = check_row0(a->row0, a->table.rows)) ||
      (rc = check_drop(a->drop, a->out.rows, &drop)))
    return rc;
  if (a->out.rows != a->tokens.count) return fail(ETC_ERR_INVALID_ARG, "out needs one row per token");
  if (a->out.cols != a->table.cols) return fail(ETC_ERR_INVALID_ARG, "out and table differ in columns");
  // an empty table has columns, an absent one none, unless there are no columns at all; no tokens need no
  // pointer to their positions
  const bool pos = a->pos_table.data || a->pos_table.cols != 0;
  if (a->tokens.count && a->out.cols && pos != (a->positions.data != nullptr))
    return fail(ETC_ERR_INVALID_ARG, "positions and pos_table go together");
  if (pos) {
    if ((rc = check_ids(a->positions, "positions")) || (rc = check_matrix(a->pos_table, "pos_table", kIn))) return rc;
    if (a->positions.count != a->tokens.count) return fail(ETC_ERR_INVALID_ARG, "positions needs one entry per token");
    if (a->pos_table.cols != a->table.cols || a->pos_table.dtype != a->table.dtype)
      return fail(ETC_ERR_INVALID_ARG, "pos_table must have the columns and dtype of table");
  }
  if (a->out.rows == 0 || a->out.cols == 0) return ETC_OK;
  return launched(etc::launch_embed(*a, drop, static_cast<hipStream_t>(stream)), "embed");
}

int etc_embed_grad_workspace(int64_t ntokens, int64_t table_rows, int64_t cols, uint64_t* bytes) {
  if (!bytes) return fail(ETC_ERR_INVALID_ARG, "bytes is NULL");
  if (ntokens < 0 || table_rows < 0 || cols < 0) return fail(ETC_ERR_INVALID_ARG, "negative size");
  if (ntokens > INT32_MAX || table_rows > INT32_MAX || cols > INT32_MAX)
    return fail(ETC_ERR_UNSUPPORTED, "more than 2^31 - 1 ids, rows or columns");
  *bytes = etc::embed_grad_sizes(uint64_t(ntokens), uint64_t(table_rows), uint64_t(cols)).total;
  return ETC_OK;
}

int etc_embed_grad(const etc_embed_grad_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  etc::Drop drop;
  int rc;
  if ((rc = check_ids(a->tokens, "tokens")) || (rc = check_matrix(a->grad, "grad", kIn)) ||
      (rc = check_matrix(a->dtable, "dtable", kOut)) || (rc = check_scale(a->scale)) ||
      (rc = check_row0(a->row0, a->dtable.rows)) ||
      (rc = check_drop(a->drop, a->grad.rows, &drop)))
    return rc;
  if (a->grad.rows != a->tokens.count) return fail(ETC_ERR_INVALID_ARG, "grad needs one row per token");
  if (a->grad.cols != a->dtable.cols) return fail(ETC_ERR_INVALID_ARG, "grad and dtable differ in columns");
  if (a->dtable.dtype != ETC_DTYPE_F32) return fail(ETC_ERR_INVALID_ARG, "dtable must be ETC_DTYPE_F32");
  if (a->reserved != 0) return fail(ETC_ERR_INVALID_ARG, "reserved must be 0");
  if (a->dtable.rows == 0 || a->dtable.cols == 0 || (a->tokens.count == 0 && a->accumulate)) return ETC_OK;
  if (!etc::embed_grad_fits(uint64_t(a->tokens.count), uint64_t(a->dtable.cols)))
    return fail(ETC_ERR_UNSUPPORTED, "too many tokens and columns for one call");
  const uint64_t need = etc::embed_grad_sizes(uint64_t(a->tokens.count), uint64_t(a->dtable.rows), uint64_t(a->dtable.cols)).total;
  if ((rc = check_workspace(a->workspace, a->workspace_bytes, need))) return rc;
  return launched(etc::launch_embed_grad(*a, drop, static_cast<hipStream_t>(stream)), "embed_grad");
}

int etc_dropout(const etc_dropout_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  etc::Drop drop;
  int rc;
  if ((rc = check_matrix(a->x, "x", kIn)) || (rc = check_like(a->out, "out", kOut, a->x)) ||
      (rc = check_drop(a->drop, a->x.rows, &drop)))
    return rc;
  if (a->bias.data && (rc = check_row(a->bias, "bias", kIn, a->x.cols, a->x.dtype))) return rc;
  if (a->residual.data && (rc = check_like(a->residual, "residual", kIn, a->x))) return rc;
  if (a->x.rows == 0 || a->x.cols == 0) return ETC_OK;
  return launched(etc::launch_dropout(*a, drop, static_cast<hipStream_t>(stream)), "dropout");
}

int etc_dropout_grad_workspace(int64_t rows, int64_t cols, uint64_t* bytes) {
  if (!bytes) return fail(ETC_ERR_INVALID_ARG, "bytes is NULL");
  if (rows < 0 || cols < 0) return fail(ETC_ERR_INVALID_ARG, "negative size");
  if (rows > INT32_MAX || cols > INT32_MAX) return fail(ETC_ERR_UNSUPPORTED, "more than 2^31 - 1 rows or columns");
  *bytes = etc::dropout_grad_bytes(uint64_t(rows), uint64_t(cols));
  return ETC_OK;
}

int etc_dropout_grad(const etc_dropout_grad_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  etc::Drop drop;
  int rc;
  if ((rc = check_matrix(a->grad, "grad", kIn)) || (rc = check_like(a->dx, "dx", kOut, a->grad)) ||
      (rc = check_drop(a->drop, a->grad.rows, &drop)))
    return rc;
  if (a->reserved != 0) return fail(ETC_ERR_INVALID_ARG, "reserved must be 0");
  if (a->dbias.data) {
    if ((rc = check_row(a->dbias, "dbias", kOut, a->grad.cols, ETC_DTYPE_F32))) return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes,
                              etc::dropout_grad_bytes(uint64_t(a->grad.rows), uint64_t(a->grad.cols)))))
      return rc;
  }
  if (a->grad.cols == 0 || (a->grad.rows == 0 && (!a->dbias.data || a->accumulate))) return ETC_OK;
  return launched(etc::launch_dropout_grad(*a, drop, static_cast<hipStream_t>(stream)), "dropout_grad");
}

int etc_adam(const etc_adam_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  if (a->count > UINT64_MAX / 8 || a->first > UINT64_MAX / 8) return fail(ETC_ERR_INVALID_ARG, "the range is too large");
  if (!(a->beta1 >= 0.0 && a->beta1 < 1.0 && a->beta2 >= 0.0 && a->beta2 < 1.0))
    return fail(ETC_ERR_INVALID_ARG, "beta1 and beta2 must lie in 0 .. 1, 1 excluded");
  if (!(a->eps >= 0.0) || !std::isfinite(a->eps) || !std::isfinite(a->lr) || !std::isfinite(a->weight_decay))
    return fail(ETC_ERR_INVALID_ARG, "lr, eps and weight_decay must be finite, eps not negative");
  if (a->step < 1) return fail(ETC_ERR_INVALID_ARG, "step counts from 1");
  const etc::AdamFactors f(*a);
  if (!std::isfinite(f.step_size) || !std::isfinite(f.decay) || !std::isfinite(f.eps) || (a->eps > 0.0 && f.eps == 0.0f))
    return fail(ETC_ERR_INVALID_ARG, "lr / (1 - beta1^step), lr * weight_decay or eps does not fit 32 bits");
  if (a->count == 0) return ETC_OK;
  for (int k = 0; k < 4; ++k) {
    if (!a->arena[k]) return fail(ETC_ERR_INVALID_ARG, "arena[%d] is NULL", k);
    if (!aligned(a->arena[k], 256)) return fail(ETC_ERR_ALIGN, "arena[%d] is not 256-byte aligned", k);
  }
  if (!a->grad) return fail(ETC_ERR_INVALID_ARG, "grad is NULL");
  if (!aligned(a->grad, 256)) return fail(ETC_ERR_ALIGN, "grad is not 256-byte aligned");
  if (!aligned(a->grad_scale, 4)) return fail(ETC_ERR_ALIGN, "grad_scale is not 4-byte aligned");
  return launched(etc::launch_adam(*a, f, static_cast<hipStream_t>(stream)), "adam");
}

}  // extern "C"
