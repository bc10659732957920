// eight.hpp -- activations in 8 bits: matrices as kernels see them, lanes'
// blocks of bytes, and the conversions from and to 32 bits.
#pragma once

#include "ops.hpp"

namespace etc {

constexpr uint32_t kWholeRow = 31;  // Mat8::shift of one scale a row: col >> 31 is 0

// Row i of the data starts at p + i * ld; the scale of column j at scale + i * sld + (j >> shift).
struct Mat8 {
  uint8_t* p;
  float* scale;
  int64_t ld, sld;
  uint32_t shift;
};

inline Mat8 mat8(const etc_matrix8& m, int64_t first_row) {
  uint32_t shift = kWholeRow;
  if (m.group) shift = uint32_t(__builtin_ctz(uint32_t(m.group)));
  return Mat8{static_cast<uint8_t*>(m.data) + first_row * m.ld, m.scale ? m.scale + first_row * m.scale_ld : nullptr, m.ld,
              m.scale_ld, shift};
}

enum Kind8 { kNone8, kInt8, kE4m3 };

inline Kind8 kind8(const etc_matrix8& m) { return m.dtype == ETC_DTYPE_E4M3 ? kE4m3 : kInt8; }

template <Kind8 k>
constexpr float kTop8 = k == kE4m3 ? 448.0f : 127.0f;
constexpr float kLeast8 = 0x1p-100f;

// The bits of |x|: ordered as whole numbers they order magnitudes, with NaN past
// the infinities, so that the largest one tells whether all are finite.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
constexpr uint32_t kInfinite = 0x7F800000u;

// From the largest magnitude's bits: the scale, and what values are multiplied with before they are rounded.
template <Kind8 k>
__device__ __forceinline__ void scale_of(uint32_t largest, float* scale, float* factor) {
  const bool fine = largest < kInfinite;
  const float a = fmaxf(__uint_as_float(fine ? largest : 0u), kLeast8);
  *scale = fine ? a / kTop8<k> : __uint_as_float(0x7FC00000u);
  *factor = fine ? kTop8<k> / a : 0.0f;
}

// kC (4, 8 or 16) bytes of a row, or the n < kC of its last block, at any
// address.  As in Raw, a row's last block is loaded as the last kC bytes of the row and
// shifted down; rows of fewer than kC columns (`shorter`) byte by byte.
template <uint32_t kC, bool kWhole>
struct Raw8 {
  static constexpr uint32_t kWords = kC / 4;
  typedef uint32_t x1 __attribute__((aligned(1)));
  typedef uint32_t x2 __attribute__((ext_vector_type(2), aligned(1)));
  typedef uint32_t x4 __attribute__((ext_vector_type(4), aligned(1)));
  uint32_t w[kWords];

  template <bool kStream = false>
  __device__ __forceinline__ void load(const uint8_t* p, uint32_t n, bool shorter) {
    if (kWhole || !shorter) {
      const uint8_t* from = kWhole ? p : p - (kC - n);
      if constexpr (kWords == 1) {
        if constexpr (kStream) w[0] = __builtin_nontemporal_load(reinterpret_cast<const x1*>(from));
        else w[0] = *reinterpret_cast<const x1*>(from);
      } else if constexpr (kWords == 2) {
        x2 v;
        if constexpr (kStream) v = __builtin_nontemporal_load(reinterpret_cast<const x2*>(from));
        else v = *reinterpret_cast<const x2*>(from);
        w[0] = v[0], w[1] = v[1];
      } else {
        x4 v;
        if constexpr (kStream) v = __builtin_nontemporal_load(reinterpret_cast<const x4*>(from));
        else v = *reinterpret_cast<const x4*>(from);
        w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
      }
    } else {  // to the same places: the upper n of kC
      zero();
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e)
        if (e + n >= kC) w[e / 4] |= uint32_t(p[e + n - kC]) << (e % 4 * 8);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) w[e] = 0;
  }
  // a last block's n bytes to the places 0 .. n - 1, zeros behind them
  __device__ __forceinline__ void shift(uint32_t n) {
    if (kWhole || n >= kC) return;
    const uint32_t s = kC - n;  // bytes to shift down
#pragma unroll
    for (uint32_t d = kWords; d; d /= 2) {
      const bool on = s & (d * 4);
#pragma unroll
      for (uint32_t e = 0; e < kWords; ++e) {
        const uint32_t here = w[e], there = e + d < kWords ? w[e + d < kWords ? e + d : e] : 0;
        w[e] = on ? there : here;
      }
    }
    const uint32_t bits = s % 4 * 8;
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) {
      const uint32_t next = e + 1 < kWords ? w[e + 1 < kWords ? e + 1 : e] : 0;
      w[e] = uint32_t((uint64_t(next) << 32 | w[e]) >> bits);
    }
  }
  // its values, unscaled
  template <Kind8 k>
  __device__ __forceinline__ void widen(float (&v)[kC], uint32_t n) const {
    Raw8 x = *this;
    x.shift(n);
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) {
      if constexpr (k == kE4m3) {
        const f32x2 low = __builtin_amdgcn_cvt_pk_f32_fp8(int(x.w[e]), false);
        const f32x2 high = __builtin_amdgcn_cvt_pk_f32_fp8(int(x.w[e]), true);
        v[4 * e] = low[0], v[4 * e + 1] = low[1], v[4 * e + 2] = high[0], v[4 * e + 3] = high[1];
      } else {
#pragma unroll
        for (uint32_t b = 0; b < 4; ++b) v[4 * e + b] = float(int32_t(x.w[e] << (24 - 8 * b)) >> 24);
      }
    }
  }
  // of v * factor, which lies within the kind's range; to nearest, ties to even.  Factor 0: zeros, whatever v holds.
  template <Kind8 k>
  __device__ __forceinline__ void narrow(const float (&v)[kC], float factor) {
#pragma unroll
    for (uint32_t e = 0; e < kWords; ++e) {
      if constexpr (k == kE4m3) {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * e] * factor, v[4 * e + 1] * factor, 0, false);
        w[e] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * e + 2] * factor, v[4 * e + 3] * factor, low, true));
      } else {
        // 1.5 * 2^23 + y has y, rounded once, in its low bits
        uint32_t q[4];
#pragma unroll
        for (uint32_t b = 0; b < 4; ++b) q[b] = __float_as_uint(__builtin_fmaf(v[4 * e + b], factor, 12582912.0f));
        const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u);
        const uint32_t high = __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu);
        w[e] = low | high;
      }
      if (factor == 0.0f) w[e] = 0;
    }
  }
  template <bool kStream = false>
  __device__ __forceinline__ void store(uint8_t* p, uint32_t n) const {
    if (kWhole || n >= kC) {
      if constexpr (kWords == 1) {
        if constexpr (kStream) __builtin_nontemporal_store(w[0], reinterpret_cast<x1*>(p));
        else *reinterpret_cast<x1*>(p) = w[0];
      } else if constexpr (kWords == 2) {
        const x2 v{w[0], w[1]};
        if constexpr (kStream) __builtin_nontemporal_store(v, reinterpret_cast<x2*>(p));
        else *reinterpret_cast<x2*>(p) = v;
      } else {
        const x4 v{w[0], w[1], w[2], w[3]};
        if constexpr (kStream) __builtin_nontemporal_store(v, reinterpret_cast<x4*>(p));
        else *reinterpret_cast<x4*>(p) = v;
      }
      return;
    }
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e)
      if (e < n) p[e] = uint8_t(w[e / 4] >> (e % 4 * 8));
  }
};

// A lane's block of kC columns in a row that a workgroup holds whole (cols >= kC).
// A row's last block is its last kC columns: the first `again` of them are the
// block's before it too.  Both lanes work out the same for those and store it, so
// nothing is shifted and stores are whole; only sums over the row leave them out.
template <uint32_t kC, bool kWhole>
struct Span {
  uint64_t at;
  uint32_t again;
  bool in;  // whether there is such a block
  __device__ __forceinline__ Span(uint64_t col, uint32_t cols) : at(col), again(0), in(col < cols) {
    if (!kWhole && in && cols - col < kC) {
      at = cols - kC;
      again = uint32_t(col - at);
    }
  }
  __device__ __forceinline__ bool counts(uint32_t e) const { return kWhole || e >= again; }
};

// The sum over a wavefront, in every lane, in an order of its own.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (uint32_t d = 1; d < 64; d *= 2) v += __shfl_xor(v, int(d));
  return v;
}
// over runs of `lanes` (a power of two) neighbouring lanes
__device__ __forceinline__ float lanes_sum(float v, uint32_t lanes) {
  for (uint32_t d = 1; d < lanes; d *= 2) v += __shfl_xor(v, int(d));
  return v;
}
// the largest over runs of `lanes` (a power of two) neighbouring lanes
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, uint32_t lanes) {
  for (uint32_t d = 1; d < lanes; d *= 2) {
    const uint32_t o = uint32_t(__shfl_xor(int(v), int(d)));
    v = o > v ? o : v;
  }
  return v;
}

// Rows of at most half a wavefront's blocks share wavefronts: the lanes of a row, or 64.
inline uint32_t lanes_of_row(uint32_t blocks) {
  uint32_t lanes = 1;
  while (lanes < blocks && lanes < 64) lanes *= 2;
  return lanes;
}
constexpr uint32_t kSharedThreads = 256;  // of a workgroup whose wavefronts have several rows each

// Calls launch(first row, rows) for runs of rows whose workgroups of `threads`, one a row, have fewer than
// 2^32 lanes, until one fails.
template <typename F>
hipError_t for_row_groups(int64_t rows, uint32_t threads, F launch) {
  const int64_t most = int64_t((uint64_t(1) << 32) - 1) / threads;
  for (int64_t at = 0; at < rows; at += most) {
    const hipError_t e = launch(at, uint32_t(rows - at < most ? rows - at : most));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
Mat<T> mat(const etc_matrix& m, int64_t first_row) {
  return Mat<T>{m.data ? static_cast<T*>(m.data) + first_row * m.ld : nullptr, m.ld};
}
template <typename T>
Mat<const T> cmat(const etc_matrix& m, int64_t first_row) {
  return Mat<const T>{m.data ? static_cast<const T*>(m.data) + first_row * m.ld : nullptr, m.ld};
}

// The launchers take checked arguments: types, sizes and strides fit.
hipError_t launch_norm(const etc_norm_args& a, hipStream_t stream);
uint64_t norm_grad_bytes(uint64_t rows, uint64_t cols);
hipError_t launch_norm_grad(const etc_norm_grad_args& a, hipStream_t stream);
hipError_t launch_store8(const etc_store8_args& a, hipStream_t stream);
hipError_t launch_load8(const etc_load8_args& a, hipStream_t stream);
hipError_t launch_matmul8(const etc_matmul8_args& a, hipStream_t stream);
hipError_t launch_rotary(const etc_rotary_args& a, hipStream_t stream);

}  // namespace etc
