// dropout.hip -- a block's epilogue, bias, dropout and residual in one pass
// (etc_dropout), and its backward with the bias's gradient (etc_dropout_grad).
//
//   out = residual + drop(x + bias);  dx = drop'(grad);  dbias (+)= column sums of drop'(grad)
//
// HBM bound: the mask is worked out from its place, so nothing but x, residual
// and out (grad and dx) is moved.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kThreads = 256;

template <typename T, bool kDrop>
__global__ __launch_bounds__(kThreads) void dropout_kernel(BlockGrid grid, Drop drop, Mat<const T> x, const T* bias,
                                                           Mat<const T> residual, Mat<T> out) {
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  if (at >= grid.n) return;
  uint32_t i, block, width;
  grid.place(at, &i, &block, &width);
  const uint64_t col = uint64_t(block) * kBlockCols;
  float v[8], b[8] = {}, r[8] = {};
  load8(x.p + int64_t(i) * x.ld + col, width, v);
  if (bias) load8(bias + col, width, b);
  if (residual.p) load8(residual.p + int64_t(i) * residual.ld + col, width, r);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += b[e];
  if (kDrop) drop.apply(i, block, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += r[e];
  store8(out.p + int64_t(i) * out.ld + col, width, v);
}

// dx, and the sums of a slab of columns over the rows [first, first + step) for the bias.
struct GradShape {
  uint32_t rows, cols, step;
};

template <typename T, bool kDrop>
__global__ __launch_bounds__(kThreads) void dropout_grad_kernel(GradShape g, Drop drop, Mat<const T> grad, Mat<T> dx,
                                                                float* partial) {
  const uint64_t col = (uint64_t(blockIdx.y) * kThreads + threadIdx.x) * kBlockCols;
  if (col >= g.cols) return;
  const uint32_t width = uint32_t(g.cols - col < kBlockCols ? g.cols - col : kBlockCols);
  const uint64_t first = uint64_t(blockIdx.x) * g.step, end = first + g.step < g.rows ? first + g.step : g.rows;
  float sum[8] = {};
  for (uint64_t i = first; i < end; ++i) {
    float v[8];
    load8(grad.p + int64_t(i) * grad.ld + col, width, v);
    if (kDrop) drop.apply(i, uint32_t(col / kBlockCols), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += v[e];
    store8(dx.p + int64_t(i) * dx.ld + col, width, v);
  }
  if (partial) store8(partial + uint64_t(blockIdx.x) * g.cols + col, width, sum);
}

__global__ __launch_bounds__(kThreads) void dbias_kernel(const float* partial, uint32_t n, uint32_t cols, float* dbias,
                                                         uint32_t accumulate) {
  const uint32_t col = blockIdx.x * kThreads + threadIdx.x;
  if (col >= cols) return;
  float sum = 0.0f;
  for (uint32_t k = 0; k < n; ++k) sum += partial[uint64_t(k) * cols + col];
  dbias[col] = (accumulate ? dbias[col] : 0.0f) + sum;
}

uint32_t grad_step(uint64_t rows) { return uint32_t(std::max<uint64_t>(32, (rows + 2047) / 2048)); }

template <typename T>
hipError_t launch_forward(const etc_dropout_args& a, const Drop& drop, hipStream_t stream) {
  return for_row_runs(a.x.rows, a.x.cols, [&](int64_t first, const BlockGrid& grid) -> hipError_t {
    auto at = [&](const etc_matrix& m) {
      return Mat<T>{m.data ? static_cast<T*>(m.data) + first * m.ld : nullptr, m.ld};
    };
    const Mat<T> x = at(a.x), r = at(a.residual), out = at(a.out);
    const T* bias = static_cast<const T*>(a.bias.data);
    Drop d = drop;
    d.row0 += uint64_t(first);
    const dim3 wgs((grid.n + kThreads - 1) / kThreads), block(kThreads);
    if (drop.limit)
      hipLaunchKernelGGL((dropout_kernel<T, true>), wgs, block, 0, stream, grid, d, Mat<const T>{x.p, x.ld}, bias,
                         Mat<const T>{r.p, r.ld}, out);
    else
      hipLaunchKernelGGL((dropout_kernel<T, false>), wgs, block, 0, stream, grid, d, Mat<const T>{x.p, x.ld}, bias,
                         Mat<const T>{r.p, r.ld}, out);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_backward(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream) {
  const uint32_t rows = uint32_t(a.grad.rows), cols = uint32_t(a.grad.cols);
  const GradShape g{rows, cols, grad_step(rows)};
  const uint32_t parts = (rows + g.step - 1) / g.step;
  float* partial = a.dbias.data ? static_cast<float*>(a.workspace) : nullptr;
  if (rows) {
    const dim3 wgs(parts, (blocks_per_row(cols) + kThreads - 1) / kThreads), block(kThreads);
    const Mat<const T> grad{static_cast<const T*>(a.grad.data), a.grad.ld};
    const Mat<T> dx{static_cast<T*>(a.dx.data), a.dx.ld};
    if (drop.limit)
      hipLaunchKernelGGL((dropout_grad_kernel<T, true>), wgs, block, 0, stream, g, drop, grad, dx, partial);
    else
      hipLaunchKernelGGL((dropout_grad_kernel<T, false>), wgs, block, 0, stream, g, drop, grad, dx, partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dbias.data) {
    hipLaunchKernelGGL(dbias_kernel, dim3((cols + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, partial, parts,
                       cols, static_cast<float*>(a.dbias.data), uint32_t(a.accumulate != 0));
  }
  return hipGetLastError();
}

}  // namespace

uint64_t dropout_grad_bytes(uint64_t rows, uint64_t cols) {
  return std::min<uint64_t>((rows + 31) / 32, 2048) * cols * sizeof(float);
}

hipError_t launch_dropout(const etc_dropout_args& a, const Drop& drop, hipStream_t stream) {
  return a.x.dtype == ETC_DTYPE_F32 ? launch_forward<float>(a, drop, stream) : launch_forward<bf16>(a, drop, stream);
}

hipError_t launch_dropout_grad(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream) {
  return a.grad.dtype == ETC_DTYPE_F32 ? launch_backward<float>(a, drop, stream)
                                       : launch_backward<bf16>(a, drop, stream);
}

}  // namespace etc
