// block.hip -- the C ABI of the operators around a block's projections
// (include/etc.h): argument checks and dispatch.  Nothing here allocates or throws.
#include <hip/hip_runtime.h>

#include <cmath>

#include "eight.hpp"
#include "etc.h"
#include "ops_check.hpp"

namespace {

int64_t scales_per_row(const etc_matrix8& m) { return m.group ? (m.cols + m.group - 1) / m.group : 1; }

// A matrix of 8-bit data that a kernel may walk.
int check_matrix8(const etc_matrix8& m, const char* what, Use use, bool scaled = true) {
  if (m.dtype != ETC_DTYPE_I8 && m.dtype != ETC_DTYPE_E4M3) return fail(ETC_ERR_INVALID_ARG, "%s: bad dtype", what);
  if (m.group != 0 && m.group != 32 && m.group != 64 && m.group != 128 && m.group != 256)
    return fail(ETC_ERR_INVALID_ARG, "%s: group must be 0, 32, 64, 128 or 256", what);
  if (m.rows < 0 || m.cols < 0) return fail(ETC_ERR_INVALID_ARG, "%s: negative size", what);
  if (m.rows > INT32_MAX || m.cols > INT32_MAX)
    return fail(ETC_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 rows or columns", what);
  if (m.rows == 0 || m.cols == 0) return ETC_OK;
  if (!m.data) return fail(ETC_ERR_INVALID_ARG, "%s is NULL", what);
  if (scaled && !m.scale) return fail(ETC_ERR_INVALID_ARG, "%s: scale is NULL", what);
  if (!aligned(m.scale, 4)) return fail(ETC_ERR_ALIGN, "%s: scale is not aligned to its elements", what);
  if (m.rows > 1) {
    if (m.ld < (use == kOut ? m.cols : 0)) return fail(ETC_ERR_INVALID_ARG, "%s: ld is too small", what);
    if (m.ld > (INT64_MAX / 8 - m.cols) / m.rows) return fail(ETC_ERR_INVALID_ARG, "%s: ld is too large", what);
    if (m.scale) {
      if (m.scale_ld < (use == kOut ? scales_per_row(m) : 0)) return fail(ETC_ERR_INVALID_ARG, "%s: scale_ld is too small", what);
      if (m.scale_ld > (INT64_MAX / 8 - m.cols) / m.rows) return fail(ETC_ERR_INVALID_ARG, "%s: scale_ld is too large", what);
    }
  }
  return ETC_OK;
}

int check_like8(const etc_matrix8& m, const char* what, Use use, const etc_matrix& x) {
  const int rc = check_matrix8(m, what, use);
  if (rc) return rc;
  if (m.rows != x.rows || m.cols != x.cols) return fail(ETC_ERR_INVALID_ARG, "%s must have the sizes of the input", what);
  return ETC_OK;
}

// Whether `out` is `in` with other distances between its rows: rows would be written over others not read yet.
bool crosses(const etc_matrix& out, const etc_matrix& in) {
  return out.data && out.data == in.data && in.rows > 1 && in.cols && out.ld != in.ld;
}

// Without elements no pointer tells that 8-bit data are given: they are what has their type and grad's sizes.
bool kept_without_elements(const etc_matrix8& m, const etc_matrix& grad) {
  return (grad.rows == 0 || grad.cols == 0) && (m.dtype == ETC_DTYPE_I8 || m.dtype == ETC_DTYPE_E4M3) && m.rows == grad.rows &&
         m.cols == grad.cols;
}

// fp32 numbers, `n` of them (none: no pointer is needed)
int check_numbers(const void* p, const char* what, int64_t n, bool needed) {
  if (n == 0 || (!p && !needed)) return ETC_OK;
  if (!p) return fail(ETC_ERR_INVALID_ARG, "%s is NULL", what);
  if (!aligned(p, 4)) return fail(ETC_ERR_ALIGN, "%s is not aligned to its elements", what);
  return ETC_OK;
}

}  // namespace

extern "C" {

int etc_norm(const etc_norm_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  int rc;
  if ((rc = check_matrix(a->x, "x", kIn))) return rc;
  if (a->x.cols && (rc = check_row(a->weight, "weight", kIn, a->x.cols, a->x.dtype))) return rc;
  if (a->residual.data && (rc = check_like(a->residual, "residual", kIn, a->x))) return rc;
  if (a->sum.data && (rc = check_like(a->sum, "sum", kOut, a->x))) return rc;
  if (a->out.data && (rc = check_like(a->out, "out", kOut, a->x))) return rc;
  if (a->out8.data) {
    if ((rc = check_like8(a->out8, "out8", kOut, a->x))) return rc;
    if (a->out8.group != 0) return fail(ETC_ERR_INVALID_ARG, "out8 must have one scale a row (group 0)");
  }
  if ((rc = check_numbers(a->rstd, "rstd", a->x.rows, false))) return rc;
  if (!(a->eps > 0.0) || !finite32(a->eps) || float(a->eps) == 0.0f)
    return fail(ETC_ERR_INVALID_ARG, "eps must be positive and finite, in 32 bits");
  if (a->x.rows == 0 || a->x.cols == 0) return ETC_OK;
  if (!a->out.data && !a->out8.data) return fail(ETC_ERR_INVALID_ARG, "out or out8 is needed");
  if (a->sum.data && a->sum.data == a->out.data) return fail(ETC_ERR_INVALID_ARG, "sum and out are the same");
  if (crosses(a->sum, a->x) || crosses(a->sum, a->residual) || crosses(a->out, a->x) || crosses(a->out, a->residual))
    return fail(ETC_ERR_INVALID_ARG, "sum and out may be x or residual itself, with its ld");
  return launched(etc::launch_norm(*a, static_cast<hipStream_t>(stream)), "norm");
}

int etc_norm_grad_workspace(int64_t rows, int64_t cols, uint64_t* bytes) {
  if (!bytes) return fail(ETC_ERR_INVALID_ARG, "bytes is NULL");
  if (rows < 0 || cols < 0) return fail(ETC_ERR_INVALID_ARG, "negative size");
  if (rows > INT32_MAX || cols > INT32_MAX) return fail(ETC_ERR_UNSUPPORTED, "more than 2^31 - 1 rows or columns");
  *bytes = etc::norm_grad_bytes(uint64_t(rows), uint64_t(cols));
  return ETC_OK;
}

int etc_norm_grad(const etc_norm_grad_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  int rc;
  if ((rc = check_matrix(a->grad, "grad", kIn)) || (rc = check_like(a->dx, "dx", kOut, a->grad))) return rc;
  if (a->grad.cols && (rc = check_row(a->weight, "weight", kIn, a->grad.cols, a->grad.dtype))) return rc;
  if (a->x.data && a->x8.data) return fail(ETC_ERR_INVALID_ARG, "x and x8 are both given");
  const bool kept = a->x8.data || (!a->x.data && kept_without_elements(a->x8, a->grad));
  if ((rc = kept ? check_like8(a->x8, "x8", kIn, a->grad) : check_like(a->x, "x", kIn, a->grad))) return rc;
  if (a->dsum.data && (rc = check_like(a->dsum, "dsum", kIn, a->grad))) return rc;
  if ((rc = check_numbers(a->rstd, "rstd", a->grad.rows, a->grad.cols != 0))) return rc;
  if (crosses(a->dx, a->grad) || crosses(a->dx, a->x) || crosses(a->dx, a->dsum))
    return fail(ETC_ERR_INVALID_ARG, "dx may be grad, x or dsum itself, with its ld");
  if (a->reserved != 0) return fail(ETC_ERR_INVALID_ARG, "reserved must be 0");
  if (a->dweight.data) {
    if ((rc = check_row(a->dweight, "dweight", kOut, a->grad.cols, ETC_DTYPE_F32))) return rc;
    if ((rc = check_workspace(a->workspace, a->workspace_bytes,
                              etc::norm_grad_bytes(uint64_t(a->grad.rows), uint64_t(a->grad.cols)))))
      return rc;
  }
  if (a->grad.cols == 0 || (a->grad.rows == 0 && (!a->dweight.data || a->accumulate))) return ETC_OK;
  return launched(etc::launch_norm_grad(*a, static_cast<hipStream_t>(stream)), "norm_grad");
}

int etc_store8(const etc_store8_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  int rc;
  if ((rc = check_matrix(a->x, "x", kIn)) || (rc = check_like8(a->out, "out", kOut, a->x)) ||
      (rc = check_numbers(a->col_scale, "col_scale", a->x.cols, false)))
    return rc;
  if (a->x.rows == 0 || a->x.cols == 0) return ETC_OK;
  return launched(etc::launch_store8(*a, static_cast<hipStream_t>(stream)), "store8");
}

int etc_load8(const etc_load8_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  int rc;
  if ((rc = check_matrix(a->out, "out", kOut)) || (rc = check_like8(a->x, "x", kIn, a->out))) return rc;
  if (a->out.rows == 0 || a->out.cols == 0) return ETC_OK;
  return launched(etc::launch_load8(*a, static_cast<hipStream_t>(stream)), "load8");
}

int etc_matmul8(const etc_matmul8_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  int rc;
  if ((rc = check_matrix8(a->x, "x", kIn, false)) || (rc = check_matrix8(a->w, "w", kIn, false)) ||
      (rc = check_matrix(a->out, "out", kOut)))
    return rc;
  if (a->x.dtype != ETC_DTYPE_I8 || a->w.dtype != ETC_DTYPE_I8) return fail(ETC_ERR_INVALID_ARG, "x and w must be ETC_DTYPE_I8");
  if (a->x.group != 0 || a->w.group != 0) return fail(ETC_ERR_INVALID_ARG, "x and w must have one scale a row (group 0)");
  if (a->x.cols != a->w.cols) return fail(ETC_ERR_INVALID_ARG, "x and w differ in columns");
  if (a->out.rows != a->x.rows || a->out.cols != a->w.rows)
    return fail(ETC_ERR_INVALID_ARG, "out needs a row for each of x's and a column for each of w's");
  if (a->x.cols > 131071) return fail(ETC_ERR_UNSUPPORTED, "more than 131071 columns of x");
  if (a->bias.data && (rc = check_row(a->bias, "bias", kIn, a->out.cols, a->out.dtype))) return rc;
  if (a->out.rows == 0 || a->out.cols == 0) return ETC_OK;
  return launched(etc::launch_matmul8(*a, static_cast<hipStream_t>(stream)), "matmul8");
}

int etc_rotary_init(etc_rotary_desc* out, int32_t dim, int32_t layout, double base, int32_t scaling, double factor,
                    double length, double low, double high) {
  if (!out) return fail(ETC_ERR_INVALID_ARG, "out is NULL");
  if (dim < 2 || dim % 2 != 0) return fail(ETC_ERR_INVALID_ARG, "dim must be even and at least 2");
  if (dim > 2 * ETC_ROTARY_PAIRS) return fail(ETC_ERR_UNSUPPORTED, "more than %d pairs", int(ETC_ROTARY_PAIRS));
  if (layout != ETC_ROTARY_HALF && layout != ETC_ROTARY_INTERLEAVED) return fail(ETC_ERR_INVALID_ARG, "bad layout");
  if (scaling < ETC_ROTARY_NONE || scaling > ETC_ROTARY_PARTS) return fail(ETC_ERR_INVALID_ARG, "bad scaling");
  if (!(base > 0.0) || !std::isfinite(base)) return fail(ETC_ERR_INVALID_ARG, "base must be positive");
  if (scaling != ETC_ROTARY_NONE && (!(factor > 0.0) || !std::isfinite(factor)))
    return fail(ETC_ERR_INVALID_ARG, "factor must be positive");
  if (scaling == ETC_ROTARY_BASE) {
    if (dim < 4) return fail(ETC_ERR_INVALID_ARG, "ETC_ROTARY_BASE needs dim 4 or more");
    base *= std::pow(factor, double(dim) / (dim - 2));
    // past 64 bits all pairs but the fastest would stand still
    if (!std::isfinite(base)) return fail(ETC_ERR_INVALID_ARG, "base * factor^(dim / (dim - 2)) is infinite");
  }
  if (scaling == ETC_ROTARY_PARTS &&
      (!(length > 0.0) || !(high > low) || !std::isfinite(length) || !std::isfinite(high - low)))
    return fail(ETC_ERR_INVALID_ARG, "length must be positive, and high above low by a finite difference");
  etc_rotary_desc d = {};
  for (int32_t j = 0; j < dim / 2; ++j) {
    double f = std::pow(base, -2.0 * j / dim);
    if (scaling == ETC_ROTARY_LINEAR) f /= factor;
    if (scaling == ETC_ROTARY_PARTS) {
      const double turns = length * f / 6.283185307179586477;
      const double u = std::fmin(1.0, std::fmax(0.0, (turns - low) / (high - low)));
      f *= u + (1.0 - u) / factor;
    }
    if (!std::isfinite(f)) return fail(ETC_ERR_INVALID_ARG, "a frequency is infinite");
    d.freq[j] = f;
  }
  d.scale = 1.0;
  d.pairs = dim / 2;
  d.layout = layout;
  *out = d;
  return ETC_OK;
}

int etc_rotary(const etc_rotary_args* a, void* stream) {
  if (!a) return fail(ETC_ERR_INVALID_ARG, "args is NULL");
  int rc;
  if ((rc = check_matrix(a->x, "x", kIn)) || (rc = check_like(a->out, "out", kOut, a->x)) ||
      (rc = check_ids(a->positions, "positions")))
    return rc;
  if (a->positions.count != a->x.rows) return fail(ETC_ERR_INVALID_ARG, "positions needs one entry per row");
  if (!a->rotary) return fail(ETC_ERR_INVALID_ARG, "rotary is NULL");
  const etc_rotary_desc& d = *a->rotary;
  if (d.pairs < 1 || d.pairs > ETC_ROTARY_PAIRS) return fail(ETC_ERR_INVALID_ARG, "rotary: pairs must lie in 1 .. %d", int(ETC_ROTARY_PAIRS));
  if (d.layout != ETC_ROTARY_HALF && d.layout != ETC_ROTARY_INTERLEAVED) return fail(ETC_ERR_INVALID_ARG, "rotary: bad layout");
  if (!finite32(d.scale)) return fail(ETC_ERR_INVALID_ARG, "rotary: scale must be finite, in 32 bits");
  for (int32_t j = 0; j < d.pairs; ++j)
    if (!std::isfinite(d.freq[j])) return fail(ETC_ERR_INVALID_ARG, "rotary: freq[%d] is not finite", int(j));
  if (a->head_dim < 2 * d.pairs) return fail(ETC_ERR_INVALID_ARG, "head_dim is below the columns that turn");
  if (a->x.cols % a->head_dim != 0) return fail(ETC_ERR_INVALID_ARG, "x's columns must be whole heads");
  if (a->x.rows == 0 || a->x.cols == 0) return ETC_OK;
  if (crosses(a->out, a->x)) return fail(ETC_ERR_INVALID_ARG, "out may be x itself, with its ld");
  return launched(etc::launch_rotary(*a, static_cast<hipStream_t>(stream)), "rotary");
}

}  // extern "C"
