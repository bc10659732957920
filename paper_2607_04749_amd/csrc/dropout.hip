// dropout.hip -- a block's epilogue, bias, dropout and residual in one pass
// (etc_dropout), and its backward with the bias's gradient (etc_dropout_grad).
//
//   out = residual + drop(x + bias);  dx = drop'(grad);  dbias (+)= column sums of drop'(grad)
//
// HBM bound: the mask is worked out from its place, so nothing but x, residual
// and out (grad and dx) is moved.  16384 x 2048 bf16, MI355X, a pass among others: the
// epilogue 31.7 us (201 MB, 6.4 TB/s), its backward 24.0 us with the bias's gradient (5.6 TB/s;
// its launches by themselves, medians of a trace, 21.2 and 4.6) and 21.8 without (6.2 TB/s).
// 1021 x 681 fp32, in graph replays: 5.4 to 5.5 us.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kFlatThreads = 64;  // elementwise launches: 31.3 us where 256 took 32.0 (16384 x 2048, bf16)
constexpr uint32_t kThreads = 256;     // launches that sum

template <typename T, bool kWhole, bool kDrop>
__global__ __launch_bounds__(kFlatThreads) void dropout_kernel(BlockGrid grid, Drop drop, Mat<const T> x, const T* bias,
                                                           Mat<const T> residual, Mat<T> out) {
  const uint32_t at = blockIdx.x * kFlatThreads + threadIdx.x;
  if (at >= grid.n) return;
  constexpr uint32_t kC = kLaneCols<T>;
  uint32_t i, block;
  grid.place(at, &i, &block);
  const uint64_t col = uint64_t(block) * kC;
  const uint32_t width = block_width<kC>(col, grid.cols);
  const bool shorter = grid.cols < kC;
  Raw<T, kC, kWhole> rx, rb, rr;
  rb.zero();
  rr.zero();
  rx.template load<true>(x.p + int64_t(i) * x.ld + col, width, shorter);
  if (residual.p) rr.template load<true>(residual.p + int64_t(i) * residual.ld + col, width, shorter);
  if (bias) rb.load(bias + col, width, shorter);
  compiler_fence();
  uint32_t bits[kC / 2];
  if (kDrop) drop.template bits<kC>(i, col, bits);  // while the loads are on their way
  float v[kC], w[kC];
  rx.widen(v, width);
  rb.widen(w, width);
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) v[e] += w[e];
  if (kDrop) drop.template apply<kC>(bits, v);
  rr.widen(w, width);
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) v[e] += w[e];
  store_block<kWhole, true>(out.p + int64_t(i) * out.ld + col, width, v);
}

// ---------------------------------------------------------------------------
// Backward with the bias's gradient.  Many rows: a workgroup has a slab of columns
// and takes rows a stride apart, kBatch per lane at a time, so that all workgroups
// together walk the matrix as one front; a lane keeps its block's sums over the
// rows that it visits, the workgroup adds its lanes' and writes one row of
// partial sums, and a second launch adds those up.

struct GradShape {
  uint32_t rows, cols;
  uint32_t lane_bits;  // 1 << lane_bits blocks of columns side by side, the other lanes further rows
  uint32_t slabs;      // slabs side by side
  uint32_t parts;      // workgroups per slab

  uint32_t down() const { return kThreads >> lane_bits; }  // rows that a workgroup visits at once
};

constexpr uint32_t kBatch = 2;     // rows in flight per lane
// Workgroups at most.  Row by row in bands of their own, 2048 workgroups took 26.3 us
// (16384 x 2048 bf16) and 60 us (fp32); as one front 26.0 and 52.0, 1024 of them
// 24.6 and 50.0, 768 24.1 and 50.2, 512 24.5 and 54.8 (dx alone 22 and 41).  3 or 4 rows
// in flight: 0.4 to 1 us more.  Non-temporal loads cost 3 us.
constexpr uint64_t kWgs = 768;
constexpr uint32_t kSlab = 64;     // blocks of a slab at most

GradShape grad_shape(uint32_t rows, uint32_t cols, uint32_t block) {
  GradShape g{rows, cols, 0, 0, 0};
  const uint32_t nb = blocks_per_row(cols, block);
  while ((1u << g.lane_bits) < std::min(nb, kSlab)) ++g.lane_bits;
  g.slabs = (nb + kSlab - 1) / kSlab;
  const uint32_t visit = g.down() * kBatch;  // rows at a time, at least 8
  g.parts = uint32_t(std::min<uint64_t>((uint64_t(rows) + visit - 1) / visit, (kWgs + g.slabs - 1) / g.slabs));
  return g;
}

template <typename T, bool kWhole, bool kDrop>
__global__ __launch_bounds__(kThreads) void dropout_grad_kernel(GradShape g, Drop drop, Mat<const T> grad, Mat<T> dx,
                                                                float* partial) {
  constexpr uint32_t kC = kLaneCols<T>;
  __shared__ float shared[kThreads][kC + 1];
  const uint32_t part = blockIdx.x / g.slabs, across = threadIdx.x & ((1u << g.lane_bits) - 1);
  const uint64_t left = uint64_t(blockIdx.x - part * g.slabs) * kSlab * kC, col = left + across * kC;
  const uint32_t width = block_width<kC>(col, g.cols);
  const uint32_t down = kThreads >> g.lane_bits;
  const bool shorter = g.cols < kC;
  float sum[kC] = {};
  if (width) {
    for (uint64_t i0 = uint64_t(part) * down * kBatch + (threadIdx.x >> g.lane_bits); i0 < g.rows;
         i0 += uint64_t(g.parts) * down * kBatch) {
      Raw<T, kC, kWhole> raw[kBatch];
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b) {
        const uint64_t i = i0 + b * down;
        raw[b].load(grad.p + int64_t(i < g.rows ? i : i0) * grad.ld + col, width, shorter);
      }
      compiler_fence();
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b) {
        const uint64_t i = i0 + b * down;
        if (i >= g.rows) break;
        uint32_t bits[kC / 2];
        if (kDrop) drop.template bits<kC>(i, col, bits);
        float v[kC];
        raw[b].widen(v, width);
        if (kDrop) drop.template apply<kC>(bits, v);
#pragma unroll
        for (uint32_t e = 0; e < kC; ++e) sum[e] += v[e];
        store_block<kWhole, true>(dx.p + int64_t(i) * dx.ld + col, width, v);
      }
    }
  }
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) shared[threadIdx.x][e] = sum[e];
  __syncthreads();
  // a column's sums lie `1 << lane_bits` lanes apart
  for (uint32_t c = threadIdx.x; c < (kC << g.lane_bits); c += kThreads) {
    float total = 0.0f;
    for (uint32_t k = 0; k < down; ++k) total += shared[(k << g.lane_bits) + c / kC][c % kC];
    if (left + c < g.cols) partial[uint64_t(part) * g.cols + left + c] = total;
  }
}

// Few rows, in one launch: a workgroup has kFewBlocks blocks of columns and all
// rows, and so the whole of its columns' sums.  Neighbours in a row, which share
// lines, are a gridDim / 8 apart, on one XCD behind one L2 (1021 x 681 fp32: 5.4 us, in
// the order of the columns 7.0).  There are few workgroups, and what they have
// in the caches grows, so up to kFewRows rows and kFewJobs blocks.  MI355X, in us, graph
// replays, one launch / two (which take 2.5 us more of the host's time):
//   rows           256         512         1021          2048
//   681 bf16    4.6 / 6.1   5.0 / 6.4    6.7 / 6.5    10.5 / 7.3
//   681 fp32    3.6 / 5.9   4.1 / 6.1    5.4 / 6.7    10.1 / 7.7
//   8192 bf16   4.9 / 8.1   5.9 / 10.3   9.1 / 12.4   14.6 / 16.7
//   8192 fp32   5.4 / 8.6   7.9 / 11.0  13.1 / 15.6   41.3 / 24.9
// Two blocks a workgroup: 8192 bf16 7.9 (256 rows); 4 rows in flight: the same.
constexpr uint32_t kFewThreads = 1024, kFewBlocks = 4, kFewDown = kFewThreads / kFewBlocks;
constexpr uint32_t kFewRows = 1024, kXcds = 8;
constexpr uint64_t kFewJobs = 1 << 21;

bool is_few(uint64_t rows, uint64_t blocks) { return rows <= kFewRows && std::max<uint64_t>(rows, 1) * blocks <= kFewJobs; }

template <typename T, bool kWhole, bool kDrop>
__global__ __launch_bounds__(kFewThreads) void dropout_grad_few_kernel(uint32_t rows, uint32_t cols, Drop drop,
                                                                       Mat<const T> grad, Mat<T> dx, float* dbias,
                                                                       uint32_t accumulate) {
  constexpr uint32_t kC = kLaneCols<T>, kWaves = kFewThreads / 64;
  __shared__ float shared[kWaves][kFewBlocks * kC];
  const uint32_t across = threadIdx.x % kFewBlocks, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t slab = blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds;
  const uint64_t left = uint64_t(slab) * kFewBlocks * kC, col = left + across * kC;
  if (left >= cols) return;
  const uint32_t width = block_width<kC>(col, cols);
  const bool shorter = cols < kC;
  // a column's sum so far, early
  const bool mine = threadIdx.x < kFewBlocks * kC && left + threadIdx.x < cols;
  float total = mine && accumulate ? dbias[left + threadIdx.x] : 0.0f;
  float sum[kC] = {};
  if (width) {
    for (uint32_t i0 = threadIdx.x / kFewBlocks; i0 < rows; i0 += kFewDown * kBatch) {
      Raw<T, kC, kWhole> raw[kBatch];
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b) {
        const uint32_t i = i0 + b * kFewDown;
        raw[b].load(grad.p + int64_t(i < rows ? i : i0) * grad.ld + col, width, shorter);
      }
      compiler_fence();
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b) {
        const uint32_t i = i0 + b * kFewDown;
        if (i >= rows) break;
        uint32_t bits[kC / 2];
        if (kDrop) drop.template bits<kC>(i, col, bits);
        float v[kC];
        raw[b].widen(v, width);
        if (kDrop) drop.template apply<kC>(bits, v);
#pragma unroll
        for (uint32_t e = 0; e < kC; ++e) sum[e] += v[e];
        store_block<kWhole>(dx.p + int64_t(i) * dx.ld + col, width, v);
      }
    }
  }
  // over the wavefront's rows, which lie kFewBlocks lanes apart, then over the wavefronts
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) {
#pragma unroll
    for (uint32_t d = kFewBlocks; d < 64; d *= 2) sum[e] += __shfl_xor(sum[e], d);
    if (lane < kFewBlocks) shared[wave][lane * kC + e] = sum[e];
  }
  __syncthreads();
  if (!mine) return;
  float all = 0.0f;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) all += shared[w][threadIdx.x];
  dbias[left + threadIdx.x] = total + all;
}

// dx alone
template <typename T, bool kWhole, bool kDrop>
__global__ __launch_bounds__(kFlatThreads) void dropout_dx_kernel(BlockGrid grid, Drop drop, Mat<const T> grad, Mat<T> dx) {
  const uint32_t at = blockIdx.x * kFlatThreads + threadIdx.x;
  if (at >= grid.n) return;
  constexpr uint32_t kC = kLaneCols<T>;
  uint32_t i, block;
  grid.place(at, &i, &block);
  const uint64_t col = uint64_t(block) * kC;
  const uint32_t width = block_width<kC>(col, grid.cols);
  const bool shorter = grid.cols < kC;
  Raw<T, kC, kWhole> raw;
  raw.template load<true>(grad.p + int64_t(i) * grad.ld + col, width, shorter);
  compiler_fence();
  uint32_t bits[kC / 2];
  if (kDrop) drop.template bits<kC>(i, col, bits);
  float v[kC];
  raw.widen(v, width);
  if (kDrop) drop.template apply<kC>(bits, v);
  store_block<kWhole, true>(dx.p + int64_t(i) * dx.ld + col, width, v);
}

// Whole lines of the partial sums: 16 columns by 64 rows read each line twice, on
// different XCDs (4096 x 8192 bf16, the whole backward: 27.3 us, so 25.8).
constexpr uint32_t kJoinCols = 32, kJoinRows = 32, kJoinBatch = 8;

__global__ __launch_bounds__(kJoinCols* kJoinRows) void dbias_kernel(const float* partial, uint32_t n, uint32_t cols,
                                                                    float* dbias, uint32_t accumulate) {
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
      dbias[col] = (accumulate ? dbias[col] : 0.0f) + sum;
    }
    __syncthreads();
  }
}

template <typename T>
hipError_t launch_forward(const etc_dropout_args& a, const Drop& drop, hipStream_t stream) {
  const bool whole = whole_blocks(a.x.cols, kLaneCols<T>);
  const auto kernel = drop.limit ? whole ? dropout_kernel<T, true, true> : dropout_kernel<T, false, true>
                                 : whole ? dropout_kernel<T, true, false> : dropout_kernel<T, false, false>;
  return for_row_runs(a.x.rows, a.x.cols, kLaneCols<T>, 1, [&](int64_t first, const BlockGrid& grid) -> hipError_t {
    auto at = [&](const etc_matrix& m) {
      return Mat<T>{m.data ? static_cast<T*>(m.data) + first * m.ld : nullptr, m.ld};
    };
    const Mat<T> x = at(a.x), r = at(a.residual), out = at(a.out);
    const T* bias = static_cast<const T*>(a.bias.data);
    Drop d = drop;
    d.row0 += uint64_t(first);
    const dim3 wgs((grid.n + kFlatThreads - 1) / kFlatThreads), block(kFlatThreads);
    hipLaunchKernelGGL(kernel, wgs, block, 0, stream, grid, d, Mat<const T>{x.p, x.ld}, bias, Mat<const T>{r.p, r.ld}, out);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_dx(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream) {
  const bool whole = whole_blocks(a.grad.cols, kLaneCols<T>);
  const auto kernel = drop.limit ? whole ? dropout_dx_kernel<T, true, true> : dropout_dx_kernel<T, false, true>
                                 : whole ? dropout_dx_kernel<T, true, false> : dropout_dx_kernel<T, false, false>;
  return for_row_runs(a.grad.rows, a.grad.cols, kLaneCols<T>, 1, [&](int64_t first, const BlockGrid& grid) -> hipError_t {
    const Mat<const T> grad{static_cast<const T*>(a.grad.data) + first * a.grad.ld, a.grad.ld};
    const Mat<T> dx{static_cast<T*>(a.dx.data) + first * a.dx.ld, a.dx.ld};
    Drop d = drop;
    d.row0 += uint64_t(first);
    const dim3 wgs((grid.n + kFlatThreads - 1) / kFlatThreads), block(kFlatThreads);
    hipLaunchKernelGGL(kernel, wgs, block, 0, stream, grid, d, grad, dx);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_backward(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream) {
  if (!a.dbias.data) return launch_dx<T>(a, drop, stream);
  if (is_few(uint64_t(a.grad.rows), blocks_per_row(a.grad.cols, kLaneCols<T>))) {
    const uint32_t rows = uint32_t(a.grad.rows), cols = uint32_t(a.grad.cols);
    const bool whole = whole_blocks(cols, kLaneCols<T>);
    const auto kernel = drop.limit ? whole ? dropout_grad_few_kernel<T, true, true> : dropout_grad_few_kernel<T, false, true>
                                   : whole ? dropout_grad_few_kernel<T, true, false> : dropout_grad_few_kernel<T, false, false>;
    const uint32_t slabs = (blocks_per_row(cols, kLaneCols<T>) + kFewBlocks - 1) / kFewBlocks;
    const dim3 wgs((slabs + kXcds - 1) / kXcds * kXcds);
    hipLaunchKernelGGL(kernel, wgs, dim3(kFewThreads), 0, stream, rows, cols, drop,
                       Mat<const T>{static_cast<const T*>(a.grad.data), a.grad.ld}, Mat<T>{static_cast<T*>(a.dx.data), a.dx.ld}, static_cast<float*>(a.dbias.data),
                       uint32_t(a.accumulate != 0));
    return hipGetLastError();
  }
  const GradShape g = grad_shape(uint32_t(a.grad.rows), uint32_t(a.grad.cols), kLaneCols<T>);
  float* partial = static_cast<float*>(a.workspace);
  if (g.parts) {
    const dim3 wgs(g.parts * g.slabs), block(kThreads);
    const Mat<const T> grad{static_cast<const T*>(a.grad.data), a.grad.ld};
    const Mat<T> dx{static_cast<T*>(a.dx.data), a.dx.ld};
    const bool whole = whole_blocks(g.cols, kLaneCols<T>);
    const auto kernel = drop.limit ? whole ? dropout_grad_kernel<T, true, true> : dropout_grad_kernel<T, false, true>
                                   : whole ? dropout_grad_kernel<T, true, false> : dropout_grad_kernel<T, false, false>;
    hipLaunchKernelGGL(kernel, wgs, block, 0, stream, g, drop, grad, dx, partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const uint32_t joins = uint32_t(std::min((uint64_t(g.cols) + kJoinCols - 1) / kJoinCols, uint64_t(1) << 16));
  hipLaunchKernelGGL(dbias_kernel, dim3(joins), dim3(kJoinCols * kJoinRows), 0, stream, partial, g.parts, g.cols,
                     static_cast<float*>(a.dbias.data), uint32_t(a.accumulate != 0));
  return hipGetLastError();
}

}  // namespace

// At most rows / 8 parts, and kWgs / slabs of them where steps are longer: it
// grows with rows and cols, so a workspace serves smaller calls.
uint64_t dropout_grad_bytes(uint64_t rows, uint64_t cols) {
  return std::min((rows + 7) / 8 * cols, kWgs * kSlab * kLaneCols<bf16> + cols) * sizeof(float);
}

hipError_t launch_dropout(const etc_dropout_args& a, const Drop& drop, hipStream_t stream) {
  return a.x.dtype == ETC_DTYPE_F32 ? launch_forward<float>(a, drop, stream) : launch_forward<bf16>(a, drop, stream);
}

hipError_t launch_dropout_grad(const etc_dropout_grad_args& a, const Drop& drop, hipStream_t stream) {
  return a.grad.dtype == ETC_DTYPE_F32 ? launch_backward<float>(a, drop, stream)
                                       : launch_backward<bf16>(a, drop, stream);
}

}  // namespace etc
