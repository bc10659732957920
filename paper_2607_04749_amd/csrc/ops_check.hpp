// ops_check.hpp -- the checks of arguments that the operators' C ABI shares.
// Each returns ETC_OK, or sets the thread's error text and returns its code.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "etc.h"
#include "etc_internal.hpp"

namespace {

int fail(int code, const char* format, ...) {
  char text[256];
  va_list args;
  va_start(args, format);
  std::vsnprintf(text, sizeof text, format, args);
  va_end(args);
  return etc::set_error(code, text);
}

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? int(ETC_OK) : fail(ETC_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

enum Use { kIn, kOut };

int64_t elem_size(int32_t dtype) { return dtype == ETC_DTYPE_BF16 ? 2 : 4; }

// A matrix that a kernel may walk: known type, sizes in 32 bits, offsets in 63.
int check_matrix(const etc_matrix& m, const char* what, Use use) {
  if (m.dtype != ETC_DTYPE_BF16 && m.dtype != ETC_DTYPE_F32) return fail(ETC_ERR_INVALID_ARG, "%s: bad dtype", what);
  if (m.reserved != 0) return fail(ETC_ERR_INVALID_ARG, "%s: reserved must be 0", what);
  if (m.rows < 0 || m.cols < 0) return fail(ETC_ERR_INVALID_ARG, "%s: negative size", what);
  if (m.rows > INT32_MAX || m.cols > INT32_MAX)
    return fail(ETC_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 rows or columns", what);
  if (m.rows == 0 || m.cols == 0) return ETC_OK;
  if (!m.data) return fail(ETC_ERR_INVALID_ARG, "%s is NULL", what);
  if (!aligned(m.data, uintptr_t(elem_size(m.dtype)))) return fail(ETC_ERR_ALIGN, "%s is not aligned to its elements", what);
  if (m.rows > 1) {
    if (m.ld < (use == kOut ? m.cols : 0)) return fail(ETC_ERR_INVALID_ARG, "%s: ld is too small", what);
    if (m.ld > (INT64_MAX / 8 - m.cols) / m.rows) return fail(ETC_ERR_INVALID_ARG, "%s: ld is too large", what);
  }
  return ETC_OK;
}

// a row of `cols` elements (the one row of a bias or its gradient)
int check_row(const etc_matrix& m, const char* what, Use use, int64_t cols, int32_t dtype) {
  const int rc = check_matrix(m, what, use);
  if (rc) return rc;
  if (m.rows != 1 || m.cols != cols) return fail(ETC_ERR_INVALID_ARG, "%s must be one row of %lld columns", what, (long long)cols);
  if (m.dtype != dtype) return fail(ETC_ERR_INVALID_ARG, "%s has another dtype than it must", what);
  return ETC_OK;
}

int check_like(const etc_matrix& m, const char* what, Use use, const etc_matrix& x) {
  const int rc = check_matrix(m, what, use);
  if (rc) return rc;
  if (m.rows != x.rows || m.cols != x.cols || m.dtype != x.dtype)
    return fail(ETC_ERR_INVALID_ARG, "%s must have the sizes and dtype of the input", what);
  return ETC_OK;
}

int check_ids(const etc_ids& v, const char* what) {
  if (v.dtype != ETC_IDS_I32 && v.dtype != ETC_IDS_I64) return fail(ETC_ERR_INVALID_ARG, "%s: bad dtype", what);
  if (v.reserved != 0) return fail(ETC_ERR_INVALID_ARG, "%s: reserved must be 0", what);
  if (v.count < 0) return fail(ETC_ERR_INVALID_ARG, "%s: negative count", what);
  if (v.count > INT32_MAX) return fail(ETC_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 ids", what);
  if (v.count == 0) return ETC_OK;
  if (!v.data) return fail(ETC_ERR_INVALID_ARG, "%s is NULL", what);
  if (!aligned(v.data, v.dtype == ETC_IDS_I64 ? 8 : 4)) return fail(ETC_ERR_ALIGN, "%s is not aligned to its elements", what);
  return ETC_OK;
}

int check_workspace(const void* p, uint64_t bytes, uint64_t need) {
  if (need == 0) return ETC_OK;
  if (!p) return fail(ETC_ERR_INVALID_ARG, "workspace is NULL");
  if (!aligned(p, 256)) return fail(ETC_ERR_ALIGN, "workspace is not 256-byte aligned");
  if (bytes < need)
    return fail(ETC_ERR_INVALID_ARG, "workspace holds %llu bytes; the call needs %llu", (unsigned long long)bytes,
                (unsigned long long)need);
  return ETC_OK;
}

// what a kernel multiplies with: an infinity would turn zeros into NaN
bool finite32(double x) { return std::isfinite(float(x)); }

int check_scale(double scale) {
  return finite32(scale) ? int(ETC_OK) : fail(ETC_ERR_INVALID_ARG, "scale must be finite, in 32 bits");
}

}  // namespace
