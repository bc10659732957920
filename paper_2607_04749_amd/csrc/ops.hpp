// ops.hpp -- what the operators of a training step share: matrices as kernels
// see them, the blocks of columns that lanes work on, and the launchers.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
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

// Accesses of 2 and 4 words at any element's address: rows of odd widths start
// anywhere, and the hardware splits what crosses a line.  The types' alignment
// holds where they are named, so no template takes them as arguments.
// kStream: non-temporal, for what is not used again by this launch.
template <typename T>
struct Words;
#define ETC_WORDS(T, A)                                                                       \
  template <>                                                                                 \
  struct Words<T> {                                                                           \
    typedef uint32_t x1 __attribute__((aligned(A)));                                          \
    typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(A)));                      \
    typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(A)));                      \
    template <bool kStream>                                                                   \
    __device__ __forceinline__ static void load2(const void* p, uint32_t* w) {                \
      x2 v;                                                                                   \
      if constexpr (kStream) v = __builtin_nontemporal_load(static_cast<const x2*>(p));       \
      else v = *static_cast<const x2*>(p);                                                    \
      w[0] = v[0], w[1] = v[1];                                                               \
    }                                                                                         \
    template <bool kStream>                                                                   \
    __device__ __forceinline__ static void load4(const void* p, uint32_t* w) {                \
      x4 v;                                                                                   \
      if constexpr (kStream) v = __builtin_nontemporal_load(static_cast<const x4*>(p));       \
      else v = *static_cast<const x4*>(p);                                                    \
      w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];                                     \
    }                                                                                         \
    template <bool kStream>                                                                   \
    __device__ __forceinline__ static void store2(void* p, const uint32_t* w) {               \
      if constexpr (kStream) __builtin_nontemporal_store(x2{w[0], w[1]}, static_cast<x2*>(p)); \
      else *static_cast<x2*>(p) = x2{w[0], w[1]};                                             \
    }                                                                                         \
    template <bool kStream>                                                                   \
    __device__ __forceinline__ static void store4(void* p, const uint32_t* w) {               \
      const x4 v{w[0], w[1], w[2], w[3]};                                                     \
      if constexpr (kStream) __builtin_nontemporal_store(v, static_cast<x4*>(p));             \
      else *static_cast<x4*>(p) = v;                                                          \
    }                                                                                         \
    __device__ __forceinline__ static void store1(void* p, uint32_t w) { *static_cast<x1*>(p) = w; } \
  }
ETC_WORDS(bf16, 2);
ETC_WORDS(float, 4);
#undef ETC_WORDS

// kC (4 or 8) elements of a row as they are in memory, or the n < kC that a row's
// last block has.  Loading and widening are apart, so that a kernel can have
// several rows' loads in flight: a value that is widened where it is loaded, on
// one side of a branch, is waited for right there.  A row's last block is loaded
// as the last kC elements of the row, and shifted when it is widened; only rows
// of fewer than kC columns (`shorter`) are loaded in pieces of 4, 2 and 1 elements,
// as all last blocks are stored.  What a last block's load reads of the block
// before is not used, so that block may be written meanwhile.  kWhole: rows of
// whole blocks only, and no code for others (whose shifts the compiler lets all
// lanes do: a lookup 26 us that takes 21). 
template <typename T, uint32_t kC, bool kWhole>
struct Raw {
  static constexpr uint32_t kWords = kC * sizeof(T) / 4;
  using E = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;
  uint32_t w[kWords];

  template <bool kStream = false>
  __device__ __forceinline__ void load(const T* p, uint32_t n, bool shorter) {
    if (kWhole || !shorter) {
      const T* from = kWhole ? p : p - (kC - n);
      if constexpr (kWords == 2) Words<T>::template load2<kStream>(from, w);
      if constexpr (kWords >= 4) Words<T>::template load4<kStream>(from, w);
      if constexpr (kWords == 8) Words<T>::template load4<kStream>(from + kC / 2, w + 4);
    } else {  // to the same places: the upper n of kC
      E x[kC] = {};
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e)
        if (e + n >= kC) x[e] = reinterpret_cast<const E*>(p)[e + n - kC];
#pragma unroll
      for (uint32_t e = 0; e < kWords; ++e) w[e] = pair(x, e);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) w[e] = 0;
  }
  __device__ __forceinline__ void widen(float (&v)[kC], uint32_t n) const {
    uint32_t x[kWords];
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) x[e] = w[e];
    if (!kWhole && n < kC) {
      const uint32_t s = kC - n;  // elements to shift down
      constexpr uint32_t per = 4 / sizeof(T);
#pragma unroll
      for (uint32_t d = kWords / 2; d; d /= 2) {
        const bool on = s & (d * per);
#pragma unroll
        for (uint32_t e = 0; e < kWords; ++e) {
          const uint32_t here = x[e], there = e + d < kWords ? x[e + d < kWords ? e + d : e] : 0;
          x[e] = on ? there : here;
        }
      }
      if constexpr (sizeof(T) == 2) {
        const uint32_t bits = s & 1 ? 16 : 0;
#pragma unroll
        for (uint32_t e = 0; e < kWords; ++e) {
          const uint32_t next = e + 1 < kWords ? x[e + 1 < kWords ? e + 1 : e] : 0;
          x[e] = uint32_t((uint64_t(next) << 32 | x[e]) >> bits);
        }
      }
    }
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) {
      if constexpr (sizeof(T) == 2) {
        v[2 * e] = __uint_as_float(x[e] << 16);
        v[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
      } else {
        v[e] = __uint_as_float(x[e]);
      }
    }
  }
  // rounds to nearest even
  __device__ __forceinline__ void narrow(const float (&v)[kC]) {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) {
      if constexpr (sizeof(T) == 2)
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * e], v[2 * e + 1]}, bf16x2));
      else
        w[e] = __float_as_uint(v[e]);
    }
  }
  template <bool kStream = false>
  __device__ __forceinline__ void store(T* p, uint32_t n) const {
    if (kWhole || n >= kC) {
      if constexpr (kWords == 2) Words<T>::template store2<kStream>(p, w);
      if constexpr (kWords >= 4) Words<T>::template store4<kStream>(p, w);
      if constexpr (kWords == 8) Words<T>::template store4<kStream>(p + kC / 2, w + 4);
      return;
    }
    // four elements where there are as many, then the last 1 to 3: their words, and where they go
    constexpr uint32_t quad = kWords * 4 / kC;
    E* q = reinterpret_cast<E*>(p);
    uint32_t x[quad];
#pragma unroll
    for (uint32_t e = 0; e < quad; ++e) {
      const uint32_t low = w[e], high = w[kWords - quad + e];  // copies: else a choice between addresses
      x[e] = n & 4 ? high : low;
    }
    if constexpr (sizeof(T) == 2) {
      if (kC == 8 && (n & 4)) Words<T>::template store2<false>(q, w);
      if (n & 2) Words<T>::store1(q + (n & 4), x[0]);
      const uint32_t a = x[0], b = x[1];
      if (n & 1) q[n & 6] = E(n & 2 ? b : a);
    } else {
      if (kC == 8 && (n & 4)) Words<T>::template store4<false>(q, w);
      if (n & 2) Words<T>::template store2<false>(q + (n & 4), x);
      const uint32_t a = x[0], b = x[2];
      if (n & 1) q[n & 6] = n & 2 ? b : a;
    }
  }

 private:
  __device__ __forceinline__ static uint32_t pair(const uint16_t (&x)[kC], uint32_t e) {
    return x[2 * e] | uint32_t(x[2 * e + 1]) << 16;
  }
  __device__ __forceinline__ static uint32_t pair(const uint32_t (&x)[kC], uint32_t e) { return x[e]; }
};

template <bool kWhole, bool kStream = false, typename T, uint32_t kC>
__device__ __forceinline__ void store_block(T* p, uint32_t n, const float (&v)[kC]) {
  Raw<T, kC, kWhole> raw;
  raw.narrow(v);
  raw.template store<kStream>(p, n);
}

// Keeps the compiler from moving memory accesses past this place: loads to
// where their values are used, which would wait for each in turn, and a store into
// other stores' place, which loses its non-temporal hint on the way.
__device__ __forceinline__ void compiler_fence() { asm volatile("" ::: "memory"); }

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

inline bool whole_blocks(int64_t cols, uint32_t block) { return cols % block == 0; }
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

// What an Adam step multiplies with, worked out in 64 bits.
struct AdamFactors {
  float beta1, rest1, beta2, rest2;  // rest = 1 - beta
  float step_size;                   // lr / (1 - beta1^t)
  float root;                        // 1 / (1 - beta2^t)
  float eps, decay;                  // decay = lr * weight_decay
  explicit AdamFactors(const etc_adam_args& x)
      : beta1(float(x.beta1)), rest1(float(1.0 - x.beta1)), beta2(float(x.beta2)), rest2(float(1.0 - x.beta2)),
        step_size(float(x.lr / (1.0 - std::pow(x.beta1, double(x.step))))),
        root(float(1.0 / (1.0 - std::pow(x.beta2, double(x.step))))), eps(float(x.eps)),
        decay(float(x.lr * x.weight_decay)) {}
};

hipError_t launch_embed(const etc_embed_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_embed_grad(const etc_embed_grad_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_dropout(const etc_dropout_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_dropout_grad(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream);
hipError_t launch_adam(const etc_adam_args& a, const AdamFactors& factors, hipStream_t stream);

}  // namespace etc
