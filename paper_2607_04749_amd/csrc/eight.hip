// eight.hip -- activations into 8 bits with scales and back (etc_store8,
// etc_load8).
//
//   scale = a / t, data = x col_scale (t / a) to nearest;  out = scale data
//
// HBM bound: x is read and the data written once, and the other way round.
// 8192 x 8192 bf16 to e4m3 in groups of 128 (206 MB): 34.6 us, 6.0 TB/s, and back 33.4 us, 6.1 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "eight.hpp"

namespace etc {

namespace {

// Rows of a lane, both on their way at once: 8192 x 8192 bf16 to e4m3 and back 67.4 us, one row 74.1,
// four 70.4; workgroups of 256 lanes 67.5 and, with one row, 75.8.
constexpr uint32_t kFlatThreads = 64, kPer = 2;
constexpr uint32_t kMostWaves = 16;
constexpr uint32_t kMostBlocks = 4;

template <typename T, uint32_t kC, bool kWhole>
__device__ __forceinline__ void load_columns(const Raw<T, kC, kWhole>& raw, const Raw<float, kC, kWhole>& factors, bool scaled,
                                             uint32_t width, float (&v)[kC]) {
  raw.widen(v, width);
  if (!scaled) return;
  float f[kC];
  factors.widen(f, width);
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) v[e] *= f[e];
}

template <uint32_t kC>
__device__ __forceinline__ uint32_t block_top(const float (&v)[kC]) {
  uint32_t top = 0;
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) top = max(top, magnitude(v[e]));
  return top;
}

// Scales of groups: a lane has a block, a group's lanes are neighbours in one
// wavefront (rows are counted in whole groups of lanes).
template <typename T, bool kWhole, Kind8 k8>
__global__ __launch_bounds__(kFlatThreads) void store8_group_kernel(BlockGrid grid, uint32_t lanes, Mat<const T> x,
                                                                    const float* col_scale, Mat8 out) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t at = blockIdx.x * kFlatThreads + threadIdx.x;
  uint32_t group = 0, block = 0;
  if (at < grid.n) grid.place(at, &group, &block);
  const uint64_t col = uint64_t(block) * kC;
  const uint32_t width = at < grid.n ? block_width<kC>(col, grid.cols) : 0;
  Raw<T, kC, kWhole> raw[kPer];
  Raw<float, kC, kWhole> factors;
  factors.zero();
#pragma unroll
  for (uint32_t r = 0; r < kPer; ++r) {
    const uint32_t i = group * kPer + r;
    raw[r].zero();
    if (width && i < grid.rows) raw[r].template load<true>(x.p + int64_t(i) * x.ld + col, width, grid.cols < kC);
  }
  if (width && col_scale) factors.load(col_scale + col, width, grid.cols < kC);
  compiler_fence();
#pragma unroll
  for (uint32_t r = 0; r < kPer; ++r) {
    const uint32_t i = group * kPer + r;
    float v[kC];
    load_columns(raw[r], factors, col_scale != nullptr, width, v);
    const uint32_t top = lanes_max(block_top(v), lanes);
    if (!width || i >= grid.rows) continue;
    float scale, factor;
    scale_of<k8>(top, &scale, &factor);
    Raw8<kC, kWhole> q;
    q.template narrow<k8>(v, factor);
    q.template store<true>(out.p + int64_t(i) * out.ld + col, width);
    if (threadIdx.x % lanes == 0) out.scale[int64_t(i) * out.sld + (col >> out.shift)] = scale;
  }
}

__device__ __forceinline__ uint32_t row_top(uint32_t top) {
  __shared__ uint32_t tops[kMostWaves];
  top = lanes_max(top, 64);
  const uint32_t waves = blockDim.x / 64;
  if (waves == 1) return top;
  if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
  __syncthreads();
  for (uint32_t w = 0; w < waves; ++w) top = max(top, tops[w]);
  return top;
}

// One scale a row: a workgroup has a row, a lane kB blocks of it.  kShared: rows of half a wavefront or less, as
// many to a workgroup as it has runs of `lanes` lanes for: 589824 rows of 128 bf16 and etc_load8 of them 87 us, and 169 with a
// wavefront each; 131072 of 256 40.9, 51.4.
template <typename T, uint32_t kB, bool kWhole, Kind8 k8, bool kShared>
__global__ __launch_bounds__(kMostWaves * 64) void store8_row_kernel(uint32_t rows, uint32_t cols, uint32_t lanes, Mat<const T> x, const float* col_scale,
                                                                     Mat8 out) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t lane = kShared ? threadIdx.x % lanes : threadIdx.x;
  const int64_t i = kShared ? blockIdx.x * (kSharedThreads / lanes) + threadIdx.x / lanes : blockIdx.x;
  if (kShared && i >= rows) return;
  auto span = [&](uint32_t b) { return Span<kC, kWhole>(uint64_t(b * blockDim.x + lane) * kC, cols); };
  Raw<T, kC, true> raw[kB];
  Raw<float, kC, true> factors[kB];
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const auto p = span(b);
    raw[b].zero();
    factors[b].zero();
    if (!p.in) continue;
    raw[b].template load<true>(x.p + i * x.ld + p.at, kC, false);
    if (col_scale) factors[b].load(col_scale + p.at, kC, false);
  }
  compiler_fence();
  float v[kB][kC];
  uint32_t top = 0;
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    load_columns(raw[b], factors[b], col_scale != nullptr, kC, v[b]);
    top = max(top, block_top(v[b]));
  }
  float scale, factor;
  if constexpr (kShared) top = lanes_max(top, lanes);
  else top = row_top(top);
  scale_of<k8>(top, &scale, &factor);
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const auto p = span(b);
    if (!p.in) continue;
    Raw8<kC, true> q;
    q.template narrow<k8>(v[b], factor);
    q.template store<true>(out.p + i * out.ld + p.at, kC);
  }
  if (lane == 0) out.scale[i * out.sld] = scale;
}

// Rows that no workgroup's registers hold, or of less than a block: read twice, the second time from the caches.
template <typename T, bool kWhole, Kind8 k8>
__global__ __launch_bounds__(kMostWaves * 64) void store8_long_kernel(uint32_t, uint32_t cols, uint32_t, Mat<const T> x, const float* col_scale,
                                                                      Mat8 out) {
  constexpr uint32_t kC = kLaneCols<T>;
  const int64_t i = blockIdx.x;
  uint32_t top = 0;
  float scale = 0.0f, factor = 0.0f;
  for (uint32_t pass = 0; pass < 2; ++pass) {
    for (uint64_t col = uint64_t(threadIdx.x) * kC; col < cols; col += uint64_t(blockDim.x) * kC) {
      const uint32_t width = block_width<kC>(col, cols);
      Raw<T, kC, kWhole> raw;
      Raw<float, kC, kWhole> factors;
      factors.zero();
      raw.load(x.p + i * x.ld + col, width, cols < kC);
      if (col_scale) factors.load(col_scale + col, width, cols < kC);
      float v[kC];
      load_columns(raw, factors, col_scale != nullptr, width, v);
      if (pass == 0) {
        top = max(top, block_top(v));
      } else {
        Raw8<kC, kWhole> q;
        q.template narrow<k8>(v, factor);
        q.store(out.p + i * out.ld + col, width);
      }
    }
    if (pass == 0) scale_of<k8>(row_top(top), &scale, &factor);
  }
  if (threadIdx.x == 0) out.scale[i * out.sld] = scale;
}

// A lane has a block of the output's columns, which lies in one group.
template <typename T, bool kWhole, Kind8 k8>
__global__ __launch_bounds__(kFlatThreads) void load8_kernel(BlockGrid grid, Mat8 x, Mat<T> out) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t at = blockIdx.x * kFlatThreads + threadIdx.x;
  if (at >= grid.n) return;
  uint32_t group, block;
  grid.place(at, &group, &block);
  const uint64_t col = uint64_t(block) * kC;
  const uint32_t width = block_width<kC>(col, grid.cols);
  Raw8<kC, kWhole> q[kPer];
  float scale[kPer];
#pragma unroll
  for (uint32_t r = 0; r < kPer; ++r) {
    const uint32_t i = min(group * kPer + r, grid.rows - 1);
    q[r].template load<true>(x.p + int64_t(i) * x.ld + col, width, grid.cols < kC);
    scale[r] = x.scale[int64_t(i) * x.sld + (col >> x.shift)];
  }
  compiler_fence();
#pragma unroll
  for (uint32_t r = 0; r < kPer; ++r) {
    const uint32_t i = group * kPer + r;
    if (i >= grid.rows) break;
    float v[kC];
    q[r].template widen<k8>(v, width);
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) v[e] *= scale[r];
    store_block<kWhole, true>(out.p + int64_t(i) * out.ld + col, width, v);
  }
}

template <typename T, bool kWhole, Kind8 k8>
hipError_t launch_store(const etc_store8_args& a, hipStream_t stream) {
  constexpr uint32_t kC = kLaneCols<T>;
  if (a.out.group) {
    const uint32_t lanes = uint32_t(a.out.group) / kC;
    const int64_t groups = (a.x.cols + a.out.group - 1) / a.out.group;
    return for_row_runs(a.x.rows, groups * a.out.group, kC, kPer, [&](int64_t first, const BlockGrid& g) -> hipError_t {
      BlockGrid grid = g;
      grid.cols = uint32_t(a.x.cols);
      hipLaunchKernelGGL((store8_group_kernel<T, kWhole, k8>), dim3((grid.n + kFlatThreads - 1) / kFlatThreads),
                         dim3(kFlatThreads), 0, stream, grid, lanes, cmat<T>(a.x, first), a.col_scale, mat8(a.out, first));
      return hipGetLastError();
    });
  }
  const uint32_t blocks = blocks_per_row(a.x.cols, kC);
  const uint32_t per = blocks <= 64 ? 1 : blocks <= 2 * 64 * kMostWaves ? 2 : kMostBlocks;
  const uint32_t waves = std::min((blocks + 64 * per - 1) / (64 * per), kMostWaves);
  const uint32_t lanes = lanes_of_row(blocks);
  const bool longer = blocks > waves * 64 * per || a.x.cols < kC, shared = !longer && lanes <= 32;
  const auto kernel = longer     ? store8_long_kernel<T, kWhole, k8>
                      : shared   ? store8_row_kernel<T, 1, kWhole, k8, true>
                      : per == 1 ? store8_row_kernel<T, 1, kWhole, k8, false>
                      : per == 2 ? store8_row_kernel<T, 2, kWhole, k8, false>
                                 : store8_row_kernel<T, kMostBlocks, kWhole, k8, false>;
  const uint32_t threads = shared ? kSharedThreads : waves * 64, at_once = shared ? kSharedThreads / lanes : 1;
  return for_row_groups(a.x.rows, threads, [&](int64_t first, uint32_t rows) -> hipError_t {
    hipLaunchKernelGGL(kernel, dim3((rows + at_once - 1) / at_once), dim3(threads), 0, stream, rows, uint32_t(a.x.cols), lanes, cmat<T>(a.x, first), a.col_scale,
                       mat8(a.out, first));
    return hipGetLastError();
  });
}

template <typename T, bool kWhole, Kind8 k8>
hipError_t launch_load(const etc_load8_args& a, hipStream_t stream) {
  return for_row_runs(a.out.rows, a.out.cols, kLaneCols<T>, kPer, [&](int64_t first, const BlockGrid& grid) -> hipError_t {
    hipLaunchKernelGGL((load8_kernel<T, kWhole, k8>), dim3((grid.n + kFlatThreads - 1) / kFlatThreads), dim3(kFlatThreads), 0,
                       stream, grid, mat8(a.x, first), mat<T>(a.out, first));
    return hipGetLastError();
  });
}

template <typename T, Kind8 k8>
hipError_t store_type(const etc_store8_args& a, hipStream_t stream) {
  return whole_blocks(a.x.cols, kLaneCols<T>) ? launch_store<T, true, k8>(a, stream) : launch_store<T, false, k8>(a, stream);
}

template <typename T, Kind8 k8>
hipError_t load_type(const etc_load8_args& a, hipStream_t stream) {
  return whole_blocks(a.out.cols, kLaneCols<T>) ? launch_load<T, true, k8>(a, stream) : launch_load<T, false, k8>(a, stream);
}

}  // namespace

hipError_t launch_store8(const etc_store8_args& a, hipStream_t stream) {
  if (a.x.dtype == ETC_DTYPE_F32)
    return kind8(a.out) == kE4m3 ? store_type<float, kE4m3>(a, stream) : store_type<float, kInt8>(a, stream);
  return kind8(a.out) == kE4m3 ? store_type<bf16, kE4m3>(a, stream) : store_type<bf16, kInt8>(a, stream);
}

hipError_t launch_load8(const etc_load8_args& a, hipStream_t stream) {
  if (a.out.dtype == ETC_DTYPE_F32)
    return kind8(a.x) == kE4m3 ? load_type<float, kE4m3>(a, stream) : load_type<float, kInt8>(a, stream);
  return kind8(a.x) == kE4m3 ? load_type<bf16, kE4m3>(a, stream) : load_type<bf16, kInt8>(a, stream);
}

}  // namespace etc
