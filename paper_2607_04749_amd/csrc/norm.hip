// norm.hip -- root-mean-square norm with the residual's addition (etc_norm).
//
//   s = x + residual;  r = 1 / sqrt(mean(s^2) + eps);  y = s r weight, in x's type, in 8 bits, or both
//
// HBM bound: x and residual are read once, s and y written once.  A row stays in
// the registers of its workgroup between the pass that sums and the one that
// multiplies.  The largest |s weight| is found beside the sum, and r times it is
// the largest |y|, so that 8 bits cost no second reduction.
// 8192 rows of 4096 bf16 with residual, sum and int8 output (235 MB): 39.1 us, 6.0 TB/s.
// One row of 4096: 3.0 us, of which 2 are the launch; the rest is two waits, for memory and for the barrier.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "eight.hpp"

namespace etc {

namespace {

constexpr uint32_t kMostWaves = 16;
constexpr uint32_t kMostBlocks = 4;  // blocks of a lane's row in registers

struct NormIn {
  uint32_t rows, cols, lanes;  // lanes of a row (kShared)
  float eps, per_col;  // 1 / cols
};

// The row's sum and largest magnitude over all wavefronts, in every lane.
template <bool kMax>
__device__ __forceinline__ void row_reduce(float* sum, uint32_t* largest) {
  __shared__ float sums[kMostWaves];
  __shared__ uint32_t tops[kMostWaves];
  *sum = wave_sum(*sum);
  if (kMax) *largest = lanes_max(*largest, 64);
  const uint32_t waves = blockDim.x / 64;
  if (waves == 1) return;
  if (threadIdx.x % 64 == 0) {
    sums[threadIdx.x / 64] = *sum;
    if (kMax) tops[threadIdx.x / 64] = *largest;
  }
  __syncthreads();
  float total = 0.0f;
  uint32_t top = 0;
  for (uint32_t w = 0; w < waves; ++w) {
    total += sums[w];
    if (kMax) top = max(top, tops[w]);
  }
  *sum = total;
  *largest = top;
}

// From the largest |s weight|: the scale of y = s weight r, and what y is multiplied with.  Rounding keeps the
// order of products with r, so that this is the largest |y|.  (r in the factor would save a product: with a small eps
// it is infinite for a row of zeros.)
template <Kind8 k>
__device__ __forceinline__ void row_scale(uint32_t largest, float r, float* scale, float* factor) {
  scale_of<k>(magnitude(r * __uint_as_float(largest)), scale, factor);
}

// A workgroup has a row, a lane kB blocks of it, one workgroup's width apart.  kShared: rows of half a wavefront or less, as
// many to a workgroup as it has lanes for: 589824 rows of 128 bf16 (query and key heads) 99 us, 6.1 TB/s, and 193 with a
// wavefront each; 131072 of 256 45.6, 50.6.
template <typename T, uint32_t kB, bool kWhole, Kind8 k8, bool kShared>
__global__ __launch_bounds__(kMostWaves * 64) void norm_kernel(NormIn in, Mat<const T> x, Mat<const T> residual,
                                                               const T* weight, Mat<T> sum, Mat<T> out, Mat8 out8,
                                                               float* rstd) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t lane = kShared ? threadIdx.x % in.lanes : threadIdx.x;
  const int64_t i = kShared ? blockIdx.x * (kSharedThreads / in.lanes) + threadIdx.x / in.lanes : blockIdx.x;
  if (kShared && i >= in.rows) return;
  auto span = [&](uint32_t b) { return Span<kC, kWhole>(uint64_t(b * blockDim.x + lane) * kC, in.cols); };
  Raw<T, kC, true> rx[kB], rr[kB], rw[kB];
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const auto p = span(b);
    rx[b].zero();
    rr[b].zero();
    rw[b].zero();
    if (!p.in) continue;
    rx[b].template load<true>(x.p + i * x.ld + p.at, kC, false);
    if (residual.p) rr[b].template load<true>(residual.p + i * residual.ld + p.at, kC, false);
    rw[b].load(weight + p.at, kC, false);
  }
  compiler_fence();
  float s[kB][kC], y[kB][kC];
  float total = 0.0f;
  uint32_t largest = 0;
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const auto p = span(b);
    float r[kC], w[kC];
    rx[b].widen(s[b], kC);
    rr[b].widen(r, kC);
    rw[b].widen(w, kC);
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) {
      s[b][e] += r[e];
      y[b][e] = s[b][e] * w[e];
      total += p.counts(e) ? s[b][e] * s[b][e] : 0.0f;
      if (k8) largest = max(largest, magnitude(y[b][e]));
    }
  }
  if constexpr (kShared) {
    total = lanes_sum(total, in.lanes);
    if (k8) largest = lanes_max(largest, in.lanes);
  } else {
    row_reduce<k8 != kNone8>(&total, &largest);
  }
  const float r = 1.0f / sqrtf(total * in.per_col + in.eps);
  if (rstd && lane == 0) rstd[i] = r;
  float factor = 0.0f;
  if (k8) {
    float scale;
    row_scale<k8 ? k8 : kInt8>(largest, r, &scale, &factor);
    if (lane == 0) out8.scale[i * out8.sld] = scale;
  }
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const auto p = span(b);
    if (!p.in) continue;
    if (sum.p) store_block<true, true>(sum.p + i * sum.ld + p.at, kC, s[b]);
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) y[b][e] *= r;
    if (k8) {
      Raw8<kC, true> q;
      q.template narrow<k8 ? k8 : kInt8>(y[b], factor);
      q.template store<true>(out8.p + i * out8.ld + p.at, kC);
    }
    if (out.p) store_block<true, true>(out.p + i * out.ld + p.at, kC, y[b]);
  }
}

// Rows that no workgroup's registers hold, or of less than a block: read twice, the second time from the
// caches.  One block after the other, so that a row may be written where it stands.
template <typename T, bool kWhole, Kind8 k8>
__global__ __launch_bounds__(kMostWaves * 64) void norm_long_kernel(NormIn in, Mat<const T> x, Mat<const T> residual,
                                                                    const T* weight, Mat<T> sum, Mat<T> out, Mat8 out8,
                                                                    float* rstd) {
  constexpr uint32_t kC = kLaneCols<T>;
  const int64_t i = blockIdx.x;
  float total = 0.0f, r = 0.0f, factor = 0.0f;
  uint32_t largest = 0;
  for (uint32_t pass = 0; pass < 2; ++pass) {
    for (uint64_t col = uint64_t(threadIdx.x) * kC; col < in.cols; col += uint64_t(blockDim.x) * kC) {
      const uint32_t width = block_width<kC>(col, in.cols);
      Raw<T, kC, kWhole> raw, rr, rw;
      rr.zero();
      raw.load(x.p + i * x.ld + col, width, in.cols < kC);
      if (residual.p) rr.load(residual.p + i * residual.ld + col, width, in.cols < kC);
      rw.load(weight + col, width, in.cols < kC);
      float s[kC], v[kC], w[kC];
      raw.widen(s, width);
      rr.widen(v, width);
      rw.widen(w, width);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) {
        s[e] += v[e];
        w[e] *= s[e];
        if (pass == 0) total += s[e] * s[e];
        if (k8 && pass == 0) largest = max(largest, magnitude(w[e]));
      }
      if (pass == 0) continue;
      if (sum.p) store_block<kWhole>(sum.p + i * sum.ld + col, width, s);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) w[e] *= r;
      if (k8) {
        Raw8<kC, kWhole> q;
        q.template narrow<k8 ? k8 : kInt8>(w, factor);
        q.store(out8.p + i * out8.ld + col, width);
      }
      if (out.p) store_block<kWhole>(out.p + i * out.ld + col, width, w);
    }
    if (pass) break;
    row_reduce<k8 != kNone8>(&total, &largest);
    r = 1.0f / sqrtf(total * in.per_col + in.eps);
    if (rstd && threadIdx.x == 0) rstd[i] = r;
    if (k8) {
      float scale;
      row_scale<k8 ? k8 : kInt8>(largest, r, &scale, &factor);
      if (threadIdx.x == 0) out8.scale[i * out8.sld] = scale;
    }
  }
}

template <typename T, bool kWhole, Kind8 k8>
hipError_t launch(const etc_norm_args& a, hipStream_t stream) {
  const uint32_t blocks = blocks_per_row(a.x.cols, kLaneCols<T>);
  // Two blocks a lane: 8192 rows of 4096 in 58.4 us with etc_load8 of them, with one block 60.1, with four
  // 58.9; a single row 3.6, 3.1 and 3.8.  Whatever the rows, so that a row has the same bits in any batch.
  const uint32_t per = blocks <= 64 ? 1 : blocks <= 2 * 64 * kMostWaves ? 2 : kMostBlocks;
  const uint32_t waves = std::min((blocks + 64 * per - 1) / (64 * per), kMostWaves);
  const uint32_t lanes = lanes_of_row(blocks);
  const bool longer = blocks > waves * 64 * per || a.x.cols < kLaneCols<T>, shared = !longer && lanes <= 32;
  const auto kernel = longer     ? norm_long_kernel<T, kWhole, k8>
                      : shared   ? norm_kernel<T, 1, kWhole, k8, true>
                      : per == 1 ? norm_kernel<T, 1, kWhole, k8, false>
                      : per == 2 ? norm_kernel<T, 2, kWhole, k8, false>
                                 : norm_kernel<T, kMostBlocks, kWhole, k8, false>;
  const uint32_t threads = shared ? kSharedThreads : waves * 64, at_once = shared ? kSharedThreads / lanes : 1;
  return for_row_groups(a.x.rows, threads, [&](int64_t first, uint32_t rows) -> hipError_t {
    const NormIn in{rows, uint32_t(a.x.cols), lanes, float(a.eps), 1.0f / float(a.x.cols)};
    hipLaunchKernelGGL(kernel, dim3((rows + at_once - 1) / at_once), dim3(threads), 0, stream, in, cmat<T>(a.x, first), cmat<T>(a.residual, first),
                       static_cast<const T*>(a.weight.data), mat<T>(a.sum, first), mat<T>(a.out, first),
                       mat8(a.out8, first), a.rstd ? a.rstd + first : nullptr);
    return hipGetLastError();
  });
}

template <typename T, bool kWhole>
hipError_t launch_kind(const etc_norm_args& a, hipStream_t stream) {
  if (!a.out8.data) return launch<T, kWhole, kNone8>(a, stream);
  return kind8(a.out8) == kE4m3 ? launch<T, kWhole, kE4m3>(a, stream) : launch<T, kWhole, kInt8>(a, stream);
}

template <typename T>
hipError_t launch_type(const etc_norm_args& a, hipStream_t stream) {
  return whole_blocks(a.x.cols, kLaneCols<T>) ? launch_kind<T, true>(a, stream) : launch_kind<T, false>(a, stream);
}

}  // namespace

hipError_t launch_norm(const etc_norm_args& a, hipStream_t stream) {
  return a.x.dtype == ETC_DTYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace etc
