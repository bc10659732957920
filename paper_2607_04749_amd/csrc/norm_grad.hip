// norm_grad.hip -- the backward of the root-mean-square norm (etc_norm_grad).
//
//   n = x r, dn = grad weight;  dx = dsum + r (dn - n mean(dn n));  dweight (+)= column sums of grad n
//
// HBM bound: grad, x (or its 8 bits) and dsum are read once and dx is written
// once.  A workgroup has a row at a time, takes rows a grid apart, and keeps its
// columns' sums in registers over them; a second launch adds the workgroups' sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "eight.hpp"

namespace etc {

namespace {

constexpr uint32_t kMostWaves = 16;
constexpr uint32_t kMostBlocks = 4;
constexpr uint32_t kAllWaves = 4096;  // wavefronts of a launch that sums

struct Shape {
  uint32_t rows, cols;
  uint32_t per, waves, parts;  // blocks of a lane, wavefronts of a row, workgroups that sum
  bool longer;                 // than the registers of a workgroup
};

Shape shape_of(uint64_t rows, uint64_t cols, uint32_t block) {
  const uint64_t blocks = (cols + block - 1) / block;
  Shape s{uint32_t(rows), uint32_t(cols), 0, 0, 0, false};
  s.per = blocks <= 64 ? 1 : blocks <= 2 * 64 * kMostWaves ? 2 : kMostBlocks;
  s.waves = uint32_t(std::min<uint64_t>((blocks + 64 * s.per - 1) / (64 * s.per), kMostWaves));
  s.longer = blocks > uint64_t(s.waves) * 64 * s.per;
  s.parts = uint32_t(std::min<uint64_t>(rows, kAllWaves / s.waves));
  return s;
}

__device__ __forceinline__ float row_sum(float sum) {
  __shared__ float sums[kMostWaves];
  sum = wave_sum(sum);
  const uint32_t waves = blockDim.x / 64;
  if (waves == 1) return sum;
  __syncthreads();  // the row before has been read
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  float total = 0.0f;
  for (uint32_t w = 0; w < waves; ++w) total += sums[w];
  return total;
}

template <typename T, bool kWhole, Kind8 k8>
struct Input {  // a block of x
  static constexpr uint32_t kC = kLaneCols<T>;
  Raw<T, kC, kWhole> raw;
  Raw8<kC, kWhole> raw8;
  float scale;

  __device__ __forceinline__ void zero() {
    if (k8) raw8.zero();
    else raw.zero();
    scale = 0.0f;
  }
  __device__ __forceinline__ void load(const Mat<const T>& x, const Mat8& x8, int64_t i, uint64_t col, uint32_t width, bool shorter) {
    if (k8) {
      raw8.template load<true>(x8.p + i * x8.ld + col, width, shorter);
      scale = x8.scale[i * x8.sld + (col >> x8.shift)];
    } else {
      raw.template load<true>(x.p + i * x.ld + col, width, shorter);
    }
  }
  // times r
  __device__ __forceinline__ void widen(float (&v)[kC], uint32_t width, float r) const {
    if constexpr (k8 != kNone8) {
      raw8.template widen<k8>(v, width);
      const float f = scale * r;
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) v[e] *= f;
    } else {
      raw.widen(v, width);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) v[e] *= r;
    }
  }
};

// n of kC fp32 sums
template <uint32_t kC, bool kWhole>
__device__ __forceinline__ void store_sums(float* p, uint32_t n, const float (&v)[kC]) {
#pragma unroll
  for (uint32_t e = 0; e < kC; e += 4) {
    if (kWhole || e + 4 <= n) {
      uint32_t w[4];
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) w[k] = __float_as_uint(v[e + k]);
      Words<float>::store4<false>(p + e, w);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k)
        if (e + k < n) p[e + k] = v[e + k];
    }
  }
}

template <typename T, uint32_t kB, bool kWhole, Kind8 k8, bool kSum>
__global__ __launch_bounds__(kMostWaves * 64) void norm_grad_kernel(uint32_t rows, uint32_t cols, float per_col, Mat<const T> grad,
                                                                    Mat<const T> x, Mat8 x8, const T* weight, Mat<const T> dsum,
                                                                    Mat<T> dx, const float* rstd, float* partial) {
  constexpr uint32_t kC = kLaneCols<T>;
  const bool shorter = cols < kC;
  Raw<T, kC, kWhole> rw[kB];
  float sums[kB][kC] = {};
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const uint64_t col = uint64_t(b * blockDim.x + threadIdx.x) * kC;
    const uint32_t width = block_width<kC>(col, cols);
    rw[b].zero();
    if (width) rw[b].load(weight + col, width, shorter);
  }
  for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int64_t i = int64_t(row);
    const float r = rstd[i];
    Raw<T, kC, kWhole> rg[kB], rd[kB];
    Input<T, kWhole, k8> rx[kB];
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const uint64_t col = uint64_t(b * blockDim.x + threadIdx.x) * kC;
      const uint32_t width = block_width<kC>(col, cols);
      rg[b].zero();
      rd[b].zero();
      rx[b].zero();
      if (!width) continue;
      rg[b].template load<true>(grad.p + i * grad.ld + col, width, shorter);
      rx[b].load(x, x8, i, col, width, shorter);
      if (dsum.p) rd[b].template load<true>(dsum.p + i * dsum.ld + col, width, shorter);
    }
    compiler_fence();
    float dot = 0.0f;
    float dn[kB][kC], n[kB][kC];
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const uint32_t width = block_width<kC>(uint64_t(b * blockDim.x + threadIdx.x) * kC, cols);
      float w[kC];
      rg[b].widen(dn[b], width);
      rx[b].widen(n[b], width, r);
      rw[b].widen(w, width);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) {
        if (kSum) sums[b][e] += dn[b][e] * n[b][e];
        dn[b][e] *= w[e];
        dot += dn[b][e] * n[b][e];
      }
    }
    const float mean = row_sum(dot) * per_col;
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const uint64_t col = uint64_t(b * blockDim.x + threadIdx.x) * kC;
      const uint32_t width = block_width<kC>(col, cols);
      if (!width) continue;
      float d[kC];
      rd[b].widen(d, width);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) d[e] += r * (dn[b][e] - n[b][e] * mean);
      store_block<kWhole, true>(dx.p + i * dx.ld + col, width, d);
    }
  }
  if (!kSum) return;
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const uint64_t col = uint64_t(b * blockDim.x + threadIdx.x) * kC;
    const uint32_t width = block_width<kC>(col, cols);
    if (width) store_sums<kC, kWhole>(partial + uint64_t(blockIdx.x) * cols + col, width, sums[b]);
  }
}

// Rows that no workgroup's registers hold: read twice, the second time from the
// caches, with the columns' sums in the workgroup's row of the workspace.
template <typename T, bool kWhole, Kind8 k8, bool kSum>
__global__ __launch_bounds__(kMostWaves * 64) void norm_grad_long_kernel(uint32_t rows, uint32_t cols, float per_col,
                                                                         Mat<const T> grad, Mat<const T> x, Mat8 x8,
                                                                         const T* weight, Mat<const T> dsum, Mat<T> dx,
                                                                         const float* rstd, float* partial) {
  constexpr uint32_t kC = kLaneCols<T>;
  for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int64_t i = int64_t(row);
    const float r = rstd[i];
    float dot = 0.0f, mean = 0.0f;
    for (uint32_t pass = 0; pass < 2; ++pass) {
      for (uint64_t col = uint64_t(threadIdx.x) * kC; col < cols; col += uint64_t(blockDim.x) * kC) {
        const uint32_t width = block_width<kC>(col, cols);
        Raw<T, kC, kWhole> rg, rd, rw;
        Input<T, kWhole, k8> rx;
        rd.zero();
        rg.load(grad.p + i * grad.ld + col, width, false);
        rx.load(x, x8, i, col, width, false);
        rw.load(weight + col, width, false);
        if (pass && dsum.p) rd.load(dsum.p + i * dsum.ld + col, width, false);
        float g[kC], n[kC], w[kC], d[kC];
        rg.widen(g, width);
        rx.widen(n, width, r);
        rw.widen(w, width);
        rd.widen(d, width);
        if (pass == 0) {
#pragma unroll
          for (uint32_t e = 0; e < kC; ++e) dot += g[e] * w[e] * n[e];
          continue;
        }
        if (kSum) {
          float* p = partial + uint64_t(blockIdx.x) * cols + col;
#pragma unroll
          for (uint32_t e = 0; e < kC; ++e)
            if (e < width) p[e] = (row == blockIdx.x ? 0.0f : p[e]) + g[e] * n[e];
        }
#pragma unroll
        for (uint32_t e = 0; e < kC; ++e) d[e] += r * (g[e] * w[e] - n[e] * mean);
        store_block<kWhole>(dx.p + i * dx.ld + col, width, d);
      }
      if (pass == 0) mean = row_sum(dot) * per_col;
    }
  }
}

// Adds the workgroups' sums, whole lines of them at a time.
constexpr uint32_t kJoinCols = 32, kJoinRows = 32, kJoinBatch = 8;

__global__ __launch_bounds__(kJoinCols* kJoinRows) void dweight_kernel(const float* partial, uint32_t n, uint32_t cols,
                                                                      float* dweight, uint32_t accumulate) {
  __shared__ float shared[kJoinRows][kJoinCols + 1];
  const uint32_t c = threadIdx.x % kJoinCols, r = threadIdx.x / kJoinCols;
  for (uint64_t first = uint64_t(blockIdx.x) * kJoinCols; first < cols; first += uint64_t(gridDim.x) * kJoinCols) {
    const uint64_t col = first + c;
    float sum = 0.0f;
    if (col < cols) {
      for (uint32_t k0 = r; k0 < n; k0 += kJoinBatch * kJoinRows) {
        float v[kJoinBatch];
#pragma unroll
        for (uint32_t b = 0; b < kJoinBatch; ++b) {
          const uint32_t k = k0 + b * kJoinRows;
          v[b] = k < n ? partial[uint64_t(k) * cols + col] : 0.0f;
        }
#pragma unroll
        for (uint32_t b = 0; b < kJoinBatch; ++b) sum += v[b];
      }
    }
    shared[r][c] = sum;
    __syncthreads();
    if (r == 0 && col < cols) {
      sum = 0.0f;
#pragma unroll
      for (uint32_t k = 0; k < kJoinRows; ++k) sum += shared[k][c];
      dweight[col] = (accumulate ? dweight[col] : 0.0f) + sum;
    }
    __syncthreads();
  }
}

template <typename T, bool kWhole, Kind8 k8, bool kSum>
hipError_t launch_rows(const etc_norm_grad_args& a, const Shape& s, hipStream_t stream) {
  const auto kernel = s.longer     ? norm_grad_long_kernel<T, kWhole, k8, kSum>
                      : s.per == 1 ? norm_grad_kernel<T, 1, kWhole, k8, kSum>
                      : s.per == 2 ? norm_grad_kernel<T, 2, kWhole, k8, kSum>
                                   : norm_grad_kernel<T, kMostBlocks, kWhole, k8, kSum>;
  const uint32_t threads = s.waves * 64;
  auto run = [&](int64_t first, uint32_t rows, uint32_t wgs) -> hipError_t {
    hipLaunchKernelGGL(kernel, dim3(wgs), dim3(threads), 0, stream, rows, s.cols, 1.0f / float(s.cols), cmat<T>(a.grad, first),
                       cmat<T>(a.x, first), mat8(a.x8, first), static_cast<const T*>(a.weight.data), cmat<T>(a.dsum, first),
                       mat<T>(a.dx, first), a.rstd + first, static_cast<float*>(a.workspace));
    return hipGetLastError();
  };
  if (kSum) return run(0, s.rows, s.parts);
  return for_row_groups(a.grad.rows, threads, [&](int64_t first, uint32_t rows) { return run(first, rows, rows); });
}

template <typename T, bool kWhole, Kind8 k8>
hipError_t launch_sum(const etc_norm_grad_args& a, hipStream_t stream) {
  const Shape s = shape_of(uint64_t(a.grad.rows), uint64_t(a.grad.cols), kLaneCols<T>);
  if (!a.dweight.data) return launch_rows<T, kWhole, k8, false>(a, s, stream);
  if (s.rows) {
    const hipError_t e = launch_rows<T, kWhole, k8, true>(a, s, stream);
    if (e != hipSuccess) return e;
  }
  const uint32_t joins = uint32_t(std::min((uint64_t(s.cols) + kJoinCols - 1) / kJoinCols, uint64_t(1) << 16));
  hipLaunchKernelGGL(dweight_kernel, dim3(joins), dim3(kJoinCols * kJoinRows), 0, stream, static_cast<const float*>(a.workspace),
                     s.parts, s.cols, static_cast<float*>(a.dweight.data), uint32_t(a.accumulate != 0));
  return hipGetLastError();
}

template <typename T, bool kWhole>
hipError_t launch_kind(const etc_norm_grad_args& a, hipStream_t stream) {
  if (a.x.data) return launch_sum<T, kWhole, kNone8>(a, stream);
  return kind8(a.x8) == kE4m3 ? launch_sum<T, kWhole, kE4m3>(a, stream) : launch_sum<T, kWhole, kInt8>(a, stream);
}

template <typename T>
hipError_t launch_type(const etc_norm_grad_args& a, hipStream_t stream) {
  return whole_blocks(a.grad.cols, kLaneCols<T>) ? launch_kind<T, true>(a, stream) : launch_kind<T, false>(a, stream);
}

}  // namespace

// At most a row a workgroup, and as many workgroups as kAllWaves have: their columns are at most
// those of their lanes, or the row's where registers do not hold it.  It grows with rows and
// cols, so a workspace serves smaller calls.
uint64_t norm_grad_bytes(uint64_t rows, uint64_t cols) {
  const uint64_t lanes = uint64_t(kAllWaves) * 64 * kMostBlocks * kLaneCols<bf16>;
  return std::min(rows * cols, std::max(lanes, kAllWaves / kMostWaves * cols)) * sizeof(float);
}

hipError_t launch_norm_grad(const etc_norm_grad_args& a, hipStream_t stream) {
  return a.grad.dtype == ETC_DTYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace etc
