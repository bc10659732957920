// ops.hpp -- what the operators of a training step share: matrices as kernels
// see them, eight-column blocks (the unit of dropout's generator and of a
// lane's work), and the launchers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "etc.h"
#include "philox.hpp"

namespace etc {

constexpr uint32_t kBlockCols = 8;  // columns of a lane's block: 16 bytes of bf16, 32 of fp32

// A matrix of T as a kernel sees it: row i starts at p + i * ld.
template <typename T>
struct Mat {
  T* p;
  int64_t ld;
};

struct Ids {
  const void* p;
  uint32_t wide;  // 64-bit ids
  __device__ __forceinline__ int64_t at(uint64_t i) const {
    return wide ? static_cast<const int64_t*>(p)[i] : int64_t(static_cast<const int32_t*>(p)[i]);
  }
};

typedef __bf16 bf16;
typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any bf16's address
typedef uint32_t u32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));  // at any fp32's
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight elements of a row as they are in memory, or the n < 8 that a row's last
// block has.  Loading and widening are apart, so that a kernel can have several
// rows' loads in flight: a value that is widened where it is loaded, on one side
// of a branch on n, is waited for right there.  Loads and stores are 16 bytes
// wide at any element's address: rows of odd widths start anywhere, and the
// hardware splits what crosses a line.  kStream: non-temporal, for what is not
// used again by this launch.
template <typename T>
struct Raw8;

template <>
struct Raw8<bf16> {
  u32x4_e2 w;
  template <bool kStream = false>
  __device__ __forceinline__ void load(const bf16* p, uint32_t n) {
    if (n >= 8) {
      const auto* q = reinterpret_cast<const u32x4_e2*>(p);
      if constexpr (kStream) w = __builtin_nontemporal_load(q);
      else w = *q;
    } else {  // elements past the end repeat the last one
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e)
        w[e] = q[2 * e < n ? 2 * e : n - 1] | uint32_t(q[2 * e + 1 < n ? 2 * e + 1 : n - 1]) << 16;
    }
  }
  __device__ __forceinline__ void zero() { w = 0; }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
};

template <>
struct Raw8<float> {
  u32x4_e4 a, b;
  template <bool kStream = false>
  __device__ __forceinline__ void load(const float* p, uint32_t n) {
    if (n >= 8) {
      const auto *q = reinterpret_cast<const u32x4_e4*>(p), *r = reinterpret_cast<const u32x4_e4*>(p + 4);
      if constexpr (kStream) a = __builtin_nontemporal_load(q), b = __builtin_nontemporal_load(r);
      else a = *q, b = *r;
    } else {
      const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        a[e] = q[e < n ? e : n - 1];
        b[e] = q[e + 4 < n ? e + 4 : n - 1];
      }
    }
  }
  __device__ __forceinline__ void zero() { a = 0, b = 0; }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = __uint_as_float(a[e]);
      v[e + 4] = __uint_as_float(b[e]);
    }
  }
};

// Rounds to nearest even, once: v holds the whole result in 32 bits.
template <bool kStream = false>
__device__ __forceinline__ void store8(bf16* p, uint32_t n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4_e2 w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * e], v[2 * e + 1]}, bf16x2));
    auto* q = reinterpret_cast<u32x4_e2*>(p);
    if constexpr (kStream) __builtin_nontemporal_store(w, q);
    else *q = w;
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e)
      if (e < n) p[e] = bf16(v[e]);
  }
}
template <bool kStream = false>
__device__ __forceinline__ void store8(float* p, uint32_t n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4_e4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = __float_as_uint(v[e]);
      b[e] = __float_as_uint(v[e + 4]);
    }
    auto *q = reinterpret_cast<u32x4_e4*>(p), *r = reinterpret_cast<u32x4_e4*>(p + 4);
    if constexpr (kStream) __builtin_nontemporal_store(a, q), __builtin_nontemporal_store(b, r);
    else *q = a, *r = b;
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e)
      if (e < n) p[e] = v[e];
  }
}

// Division of n < 2^31 by d >= 1 as a product (Granlund and Montgomery, "Division
// by Invariant Integers using Multiplication", PLDI 1994): q = (hi(n m) + n) >> s.
struct Divisor {
  uint32_t d, m, s;
  Divisor() = default;
  explicit Divisor(uint32_t by) : d(by), m(0), s(0) {
    while (s < 32 && (uint64_t(1) << s) < by) ++s;
    m = uint32_t(((uint64_t(1) << 32) * ((uint64_t(1) << s) - by)) / by + 1);
  }
  __host__ __device__ uint32_t div(uint32_t n) const { return uint32_t((((uint64_t(n) * m) >> 32) + n) >> s); }
};

inline uint32_t blocks_per_row(int64_t cols) { return uint32_t((cols + kBlockCols - 1) / kBlockCols); }

// An elementwise launch: a lane has one eight-column block of `per` consecutive
// rows.  Lanes are numbered along the row, then down the groups of rows.
struct BlockGrid {
  uint32_t n;  // lanes with work, < 2^31
  uint32_t rows, cols;
  Divisor per_row;
  // lane `at`: its group of rows, its block's number in the row, and how many columns that has
  __device__ __forceinline__ void place(uint32_t at, uint32_t* group, uint32_t* block, uint32_t* width) const {
    *group = per_row.div(at);
    *block = at - *group * per_row.d;
    const uint32_t left = cols - *block * kBlockCols;
    *width = left < kBlockCols ? left : kBlockCols;
  }
};

// Calls launch(first row, grid) for runs of rows of fewer than 2^31 lanes, until one fails.
template <typename F>
hipError_t for_row_runs(int64_t rows, int64_t cols, uint32_t per, F launch) {
  const uint32_t nb = blocks_per_row(cols);
  const int64_t most = INT32_MAX / int64_t(nb) * per;
  for (int64_t at = 0; at < rows; at += most) {
    const int64_t n = rows - at < most ? rows - at : most;
    const hipError_t e = launch(at, BlockGrid{uint32_t((n + per - 1) / per) * nb, uint32_t(n), uint32_t(cols), Divisor(nb)});
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The launchers take checked arguments: types, sizes and strides fit.
struct EmbedGradSizes {
  uint64_t keys[2], order[2], parts;  // byte offsets in the workspace
  uint64_t total;                             // its length
};
EmbedGradSizes embed_grad_sizes(uint64_t ntokens, uint64_t rows, uint64_t cols);
// whether a call's launches are within the 2^32 lanes that a grid may have
bool embed_grad_fits(uint64_t ntokens, uint64_t cols);
uint64_t dropout_grad_bytes(uint64_t rows, uint64_t cols);

hipError_t launch_embed(const etc_embed_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_embed_grad(const etc_embed_grad_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_dropout(const etc_dropout_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_dropout_grad(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_adam(const etc_adam_args& a, hipStream_t stream);

}  // namespace etc
