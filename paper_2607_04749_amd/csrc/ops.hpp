// ops.hpp -- what the operators of a training step share: matrices as kernels
// see them, the blocks of columns that lanes work on, and the launchers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "etc.h"
#include "philox.hpp"

namespace etc {

// Columns of a lane's block: 16 bytes of the type that a kernel mostly moves,
// so that a wavefront's accesses cover whole lines one after the other.  Lanes of
// eight fp32 columns, two accesses 32 bytes apart each, reached 3.8 TB/s in the
// dropout backward where bf16 reached 5.0.
template <typename T>
constexpr uint32_t kLaneCols = 16 / sizeof(T);

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
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Words at any element's address: rows of odd widths start anywhere, and the
// hardware splits what crosses a line.
template <typename T>
struct Words;
template <>
struct Words<bf16> {
  typedef uint32_t x1 __attribute__((aligned(2)));
  typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(2)));
  typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct Words<float> {
  typedef uint32_t x1;
  typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(4)));
  typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(4)));
};

// kC (4 or 8) elements of a row as they are in memory, or the n < kC that a row's
// last block has.  Loading and widening are apart, so that a kernel can have
// several rows' loads in flight: a value that is widened where it is loaded, on
// one side of a branch on n, is waited for right there.  A last block moves in
// pieces of 4, 2 and 1 elements.  kStream: non-temporal, for what is not used
// again by this launch.
template <typename T, uint32_t kC>
struct Raw;

template <uint32_t kC>
struct Raw<bf16, kC> {
  static constexpr uint32_t kWords = kC / 2;
  uint32_t w[kWords];
  template <bool kStream = false>
  __device__ __forceinline__ void load(const bf16* p, uint32_t n) {
    using V = typename std::conditional<kC == 8, Words<bf16>::x4, Words<bf16>::x2>::type;
    if (n >= kC) {
      const V* q = reinterpret_cast<const V*>(p);
      V v;
      if constexpr (kStream) v = __builtin_nontemporal_load(q);
      else v = *q;
#pragma unroll
      for (uint32_t e = 0; e < kWords; ++e) w[e] = v[e];
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
      Words<bf16>::x2 four = 0;
      uint32_t two = 0, one = 0;
      if (kC == 8 && (n & 4)) four = *reinterpret_cast<const Words<bf16>::x2*>(q);
      if (n & 2) two = *reinterpret_cast<const Words<bf16>::x1*>(q + (n & 4));
      if (n & 1) one = q[n & 6];
      const uint32_t low = n & 2 ? two : one, high = n & 2 ? one : 0;  // the last 1 to 3
      const uint32_t f0 = four[0], f1 = four[1];
      w[0] = n & 4 ? f0 : low;
      w[1] = n & 4 ? f1 : high;
      if constexpr (kC == 8) w[2] = low, w[3] = high;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) w[e] = 0;
  }
  __device__ __forceinline__ void widen(float (&v)[kC]) const {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
  // rounds to nearest even
  __device__ __forceinline__ void narrow(const float (&v)[kC]) {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e)
      w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * e], v[2 * e + 1]}, bf16x2));
  }
  template <bool kStream = false>
  __device__ __forceinline__ void store(bf16* p, uint32_t n) const {
    using V = typename std::conditional<kC == 8, Words<bf16>::x4, Words<bf16>::x2>::type;
    if (n >= kC) {
      V v;
#pragma unroll
      for (uint32_t e = 0; e < kWords; ++e) v[e] = w[e];
      V* q = reinterpret_cast<V*>(p);
      if constexpr (kStream) __builtin_nontemporal_store(v, q);
      else *q = v;
    } else {
      uint16_t* q = reinterpret_cast<uint16_t*>(p);
      if (kC == 8 && (n & 4)) *reinterpret_cast<Words<bf16>::x2*>(q) = Words<bf16>::x2{w[0], w[1]};
      // copies: a choice between elements of an array would be one between their addresses
      const uint32_t w0 = w[0], w1 = w[1], w2 = w[kWords - 2], w3 = w[kWords - 1];
      const uint32_t low = n & 4 ? w2 : w0, high = n & 4 ? w3 : w1;
      if (n & 2) *reinterpret_cast<Words<bf16>::x1*>(q + (n & 4)) = low;
      if (n & 1) q[n & 6] = uint16_t(n & 2 ? high : low);
    }
  }
};

template <uint32_t kC>
struct Raw<float, kC> {
  uint32_t w[kC];
  template <bool kStream = false>
  __device__ __forceinline__ void load(const float* p, uint32_t n) {
    using V = Words<float>::x4;
    if (n >= kC) {
#pragma unroll
      for (uint32_t h = 0; h < kC / 4; ++h) {
        const V* q = reinterpret_cast<const V*>(p + 4 * h);
        V v;
        if constexpr (kStream) v = __builtin_nontemporal_load(q);
        else v = *q;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) w[4 * h + e] = v[e];
      }
    } else {
      const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
      V four = 0;
      Words<float>::x2 two = 0;
      uint32_t one = 0;
      if (kC == 8 && (n & 4)) four = *reinterpret_cast<const V*>(q);
      if (n & 2) two = *reinterpret_cast<const Words<float>::x2*>(q + (n & 4));
      if (n & 1) one = q[n & 6];
      const uint32_t tail[4] = {n & 2 ? two[0] : one, two[1], one, 0};  // the last 1 to 3
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t f = four[e], t = tail[e];
        w[e] = n & 4 ? f : t;
        if constexpr (kC == 8) w[4 + e] = t;
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) w[e] = 0;
  }
  __device__ __forceinline__ void widen(float (&v)[kC]) const {
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) v[e] = __uint_as_float(w[e]);
  }
  __device__ __forceinline__ void narrow(const float (&v)[kC]) {
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) w[e] = __float_as_uint(v[e]);
  }
  template <bool kStream = false>
  __device__ __forceinline__ void store(float* p, uint32_t n) const {
    using V = Words<float>::x4;
    if (n >= kC) {
#pragma unroll
      for (uint32_t h = 0; h < kC / 4; ++h) {
        const V v{w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
        V* q = reinterpret_cast<V*>(p + 4 * h);
        if constexpr (kStream) __builtin_nontemporal_store(v, q);
        else *q = v;
      }
    } else {
      uint32_t* q = reinterpret_cast<uint32_t*>(p);
      if (kC == 8 && (n & 4)) *reinterpret_cast<V*>(q) = V{w[0], w[1], w[2], w[3]};
      // copies: a choice between elements of an array would be one between their addresses
      const uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w4 = w[kC - 4], w5 = w[kC - 3], w6 = w[kC - 2];
      const uint32_t t0 = n & 4 ? w4 : w0, t1 = n & 4 ? w5 : w1, t2 = n & 4 ? w6 : w2;
      if (n & 2) *reinterpret_cast<Words<float>::x2*>(q + (n & 4)) = Words<float>::x2{t0, t1};
      if (n & 1) q[n & 6] = n & 2 ? t2 : t0;
    }
  }
};

template <bool kStream = false, typename T, uint32_t kC>
__device__ __forceinline__ void store_block(T* p, uint32_t n, const float (&v)[kC]) {
  Raw<T, kC> raw;
  raw.narrow(v);
  raw.template store<kStream>(p, n);
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

inline uint32_t blocks_per_row(int64_t cols, uint32_t block) { return uint32_t((cols + block - 1) / block); }

// Columns of the block of kC that begins at `col`, 0 past the matrix.
template <uint32_t kC>
__device__ __forceinline__ uint32_t block_width(uint64_t col, uint32_t cols) {
  return col >= cols ? 0 : cols - col < kC ? uint32_t(cols - col) : kC;
}

// An elementwise launch: a lane has one block of `per` consecutive rows.
// Lanes are numbered along the row, then down the groups of rows.
struct BlockGrid {
  uint32_t n;  // lanes with work, < 2^31
  uint32_t rows, cols;
  Divisor per_row;
  // lane `at`: its group of rows and its block's number in the row
  __device__ __forceinline__ void place(uint32_t at, uint32_t* group, uint32_t* block) const {
    *group = per_row.div(at);
    *block = at - *group * per_row.d;
  }
};

// Calls launch(first row, grid) for runs of rows of fewer than 2^31 lanes, until one fails.
template <typename F>
hipError_t for_row_runs(int64_t rows, int64_t cols, uint32_t block, uint32_t per, F launch) {
  const uint32_t nb = blocks_per_row(cols, block);
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
