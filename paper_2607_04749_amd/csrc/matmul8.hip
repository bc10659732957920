// matmul8.hip -- products of 8-bit integers with a scale for each row of either
// operand (etc_matmul8).
//
//   out[m, n] = sx[m] sw[n] (sum over k of x[m, k] w[n, k]) + bias[n]
//
// The sums are exact in 32-bit integers, so how they are split changes no bit.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "eight.hpp"

namespace etc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Product {
  const uint8_t *x, *w;
  int64_t xld, wld;
  const float *sx, *sw;
  int64_t sxld, swld;  // from a row's scale to the next one's
  uint32_t m, n, k;
  void* out;
  int64_t ld;
  const void* bias;
};

template <typename T>
__device__ __forceinline__ float widened(const void* p, uint32_t j) {
  return float(static_cast<const T*>(p)[j]);
}

// 64 x 64 of the output by four wavefronts, any sizes, strides and alignment.
constexpr uint32_t kTile = 64, kStep = 64, kPad = 16;

template <typename T>
__global__ __launch_bounds__(256) void matmul8_any_kernel(Product p, uint32_t tiles_n) {
  __shared__ __attribute__((aligned(16))) uint8_t xs[kTile][kStep + kPad], ws[kTile][kStep + kPad];
  const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const uint64_t m0 = uint64_t(tm) * kTile, n0 = uint64_t(tn) * kTile;
  const uint32_t row = threadIdx.x / 4, part = threadIdx.x % 4 * 16;
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  i32x4 acc[4] = {};
  for (uint32_t k0 = 0; k0 < p.k; k0 += kStep) {
    Raw8<16, false> rx, rw;
    rx.zero();
    rw.zero();
    const uint32_t width = block_width<16>(uint64_t(k0) + part, p.k);
    if (width) {
      if (m0 + row < p.m) rx.load(p.x + int64_t(m0 + row) * p.xld + k0 + part, width, p.k < 16);
      if (n0 + row < p.n) rw.load(p.w + int64_t(n0 + row) * p.wld + k0 + part, width, p.k < 16);
      rx.shift(width);
      rw.shift(width);
    }
    __syncthreads();
    *reinterpret_cast<i32x4*>(&xs[row][part]) = i32x4{int(rx.w[0]), int(rx.w[1]), int(rx.w[2]), int(rx.w[3])};
    *reinterpret_cast<i32x4*>(&ws[row][part]) = i32x4{int(rw.w[0]), int(rw.w[1]), int(rw.w[2]), int(rw.w[3])};
    __syncthreads();
    const i32x4 b = *reinterpret_cast<const i32x4*>(&xs[wave * 16 + lane % 16][lane / 16 * 16]);
#pragma unroll
    for (uint32_t t = 0; t < 4; ++t) {
      const i32x4 a = *reinterpret_cast<const i32x4*>(&ws[t * 16 + lane % 16][lane / 16 * 16]);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc[t], 0, 0, 0);
    }
  }
  const uint64_t m = m0 + wave * 16 + lane % 16;
  if (m >= p.m) return;
  const float sx = p.sx ? p.sx[int64_t(m) * p.sxld] : 1.0f;
#pragma unroll
  for (uint32_t t = 0; t < 4; ++t) {
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint64_t n = n0 + t * 16 + lane / 16 * 4 + e;
      if (n >= p.n) continue;
      float v = float(acc[t][e]) * sx * (p.sw ? p.sw[int64_t(n) * p.swld] : 1.0f);
      if (p.bias) v += widened<T>(p.bias, uint32_t(n));
      static_cast<T*>(p.out)[int64_t(m) * p.ld + int64_t(n)] = T(v);
    }
  }
}

template <typename T>
hipError_t launch_type(const etc_matmul8_args& a, hipStream_t stream) {
  const uint32_t tiles_n = uint32_t((a.out.cols + kTile - 1) / kTile);
  const int64_t most = INT32_MAX / 256 / tiles_n * int64_t(kTile);  // rows of a launch
  if (most == 0) return hipErrorInvalidValue;
  for (int64_t at = 0; at < a.out.rows; at += most) {
    const Mat8 x = mat8(a.x, at), w = mat8(a.w, 0);
    const uint32_t rows = uint32_t(std::min(most, a.out.rows - at));
    const Product p{x.p, w.p, x.ld, w.ld, x.scale, w.scale, x.sld, w.sld, rows, uint32_t(a.out.cols), uint32_t(a.x.cols),
                    mat<T>(a.out, at).p, a.out.ld, a.bias.data};
    hipLaunchKernelGGL(matmul8_any_kernel<T>, dim3((rows + kTile - 1) / kTile * tiles_n), dim3(256), 0, stream, p, tiles_n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_matmul8(const etc_matmul8_args& a, hipStream_t stream) {
  return a.out.dtype == ETC_DTYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace etc
