// norm_grad.hip -- the backward of the root-mean-square norm (etc_norm_grad).
//
//   n = x r, dn = grad weight;  dx = dsum + r (dn - n mean(dn n));  dweight (+)= column sums of grad n
//
// HBM bound: grad, x (or its 8 bits) and dsum are read once and dx is written
// once.  A workgroup has a row at a time, takes rows a grid apart, and keeps its
// columns' sums in registers over them; a second launch adds the workgroups' sums.
// 8192 rows of 4096 bf16, x in int8, dsum (235 MB): 40.8 us, 6.0 TB/s with the sums, then 4.6 us for the
// 8 MB of sums.  The next row's loads before this one's barrier took the registers of half the
// wavefronts and were slower; one barrier a row, with its sums in turn, is what is left of the wait.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "eight.hpp"

namespace etc {

namespace {

constexpr uint32_t kMostWaves = 16;
constexpr uint32_t kMostBlocks = 2;
constexpr uint32_t kCus = 256;
constexpr uint32_t kAllWaves = 4096;  // wavefronts of a launch that sums
// Rows of a workgroup at least: its sums take as much to write and read again as a row does.  2048 x 681
// bf16, in us: 13.5 with one, 11.3 with two, 11.5 with four, 15.4 with eight.
constexpr uint32_t kRowsAPart = 4;

struct Shape {
  uint32_t rows, cols;
  uint32_t per, waves, parts;  // blocks of a lane, wavefronts of a row, workgroups that sum
  uint32_t lanes, joined;      // of a row within a wavefront, or 0: longer ones; wavefronts whose sums a workgroup joins
  bool longer;                 // than the registers of a workgroup, or less than a block
};

Shape shape_of(uint64_t rows, uint64_t cols, uint32_t block) {
  const uint64_t blocks = (cols + block - 1) / block;
  Shape s{uint32_t(rows), uint32_t(cols), 0, 0, 0, 0, 1, false};
  s.per = blocks <= 64 * kMostWaves ? 1 : kMostBlocks;
  s.waves = uint32_t(std::min<uint64_t>((blocks + 64 * s.per - 1) / (64 * s.per), kMostWaves));
  s.longer = blocks > uint64_t(s.waves) * 64 * s.per || cols < block;
  uint64_t of_part = kRowsAPart;
  if (!s.longer && blocks <= 64) {
    s.lanes = lanes_of_row(uint32_t(blocks));
    of_part *= 64 / s.lanes;
    // as few sums as leave each CU a workgroup
    s.joined = rows >= of_part * 16 * kCus ? 16 : rows >= of_part * 4 * kCus ? 4 : 1;
    of_part *= s.joined;
  }
  s.parts = uint32_t(std::min<uint64_t>((rows + of_part - 1) / of_part, kAllWaves / (s.waves * s.joined)));
  return s;
}

// The sum over the `waves` wavefronts that share a row; all wavefronts of the
// workgroup call it, with `turn` 0 and 1 in turn: who writes a turn's sums has passed the barrier of the other
// turn, before which all have read this one's.
__device__ __forceinline__ float row_sum(float sum, uint32_t waves, uint32_t turn) {
  __shared__ float sums[2][kMostWaves];
  sum = wave_sum(sum);
  if (blockDim.x == 64) return sum;
  if (threadIdx.x % 64 == 0) sums[turn][threadIdx.x / 64] = sum;
  __syncthreads();
  const uint32_t first = threadIdx.x / 64 / waves * waves;
  float total = 0.0f;
  for (uint32_t w = 0; w < waves; ++w) total += sums[turn][min(first + w, kMostWaves - 1)];
  return total;
}

template <typename T, bool kWhole, Kind8 k8>
struct Input {  // a block of x
  static constexpr uint32_t kC = kLaneCols<T>;
  Raw<T, kC, kWhole> raw;
  Raw8<kC, kWhole> raw8;
  float scale, before;  // of the block's last column; of its first ones, which may be of the group before
  uint32_t again = 0;   // how many of those there are

  __device__ __forceinline__ void zero() {
    if (k8) raw8.zero();
    else raw.zero();
    scale = before = 0.0f;
  }
  __device__ __forceinline__ void load(const Mat<const T>& x, const Mat8& x8, int64_t i, uint64_t col, uint32_t width, bool shorter) {
    if (k8) {
      raw8.template load<true>(x8.p + i * x8.ld + col, width, shorter);
      scale = x8.scale[i * x8.sld + (col >> x8.shift)];
    } else {
      raw.template load<true>(x.p + i * x.ld + col, width, shorter);
    }
  }
  template <bool kAll>
  __device__ __forceinline__ void load(const Mat<const T>& x, const Mat8& x8, int64_t i, const Span<kC, kAll>& p) {
    load(x, x8, i, p.at, kC, false);
    if (kAll || !k8) return;
    again = p.again;
    before = scale;
    scale = x8.scale[i * x8.sld + ((p.at + kC - 1) >> x8.shift)];
  }
  // times r
  __device__ __forceinline__ void widen(float (&v)[kC], uint32_t width, float r) const {
    if constexpr (k8 != kNone8) {
      raw8.template widen<k8>(v, width);
      const float f = scale * r, f0 = before * r;
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) v[e] *= e < again ? f0 : f;
    } else {
      raw.widen(v, width);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) v[e] *= r;
    }
  }
};

// Where one launch takes less than two: its workgroups of columns read all rows again, from the caches, and
// have to be done before the others.  In us, with one launch and with two: 1021 rows of 681 fp32 8.5, 9.7; bf16:
// 256 of 681 5.3, 8.3; 512 of 8192 13.5, 16.8; 1024 of 2048 10.7, 11.3.
bool is_few(const Shape& s) { return s.rows && !s.longer && s.rows <= 1024 && (s.per == 1 || s.rows <= 128); }

// kC fp32 sums
template <uint32_t kC>
__device__ __forceinline__ void store_sums(float* p, const float (&v)[kC]) {
#pragma unroll
  for (uint32_t e = 0; e < kC; e += 4) {
    uint32_t w[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) w[k] = __float_as_uint(v[e + k]);
    Words<float>::store4<false>(p + e, w);
  }
}

struct In {
  uint32_t rows, cols;
  float per_col;  // 1 / cols
  uint32_t lanes;  // of a row (kShared)
};

// Lane `lane` of the `lanes` that share a row: kB blocks of it, `lanes` blocks apart.
template <typename T, uint32_t kB, bool kWhole, Kind8 k8>
struct Row {
  static constexpr uint32_t kC = kLaneCols<T>;
  typedef Raw<T, kC, true> Block;
  Block grad[kB], dsum[kB];
  Input<T, true, k8> x[kB];
  float r;

  __device__ __forceinline__ static Span<kC, kWhole> span(const In& in, uint32_t b, uint32_t lane, uint32_t lanes) {
    return Span<kC, kWhole>(uint64_t(b * lanes + lane) * kC, in.cols);
  }

  __device__ __forceinline__ static void load_weight(const In& in, uint32_t lane, uint32_t lanes, const T* weight, Block (&w)[kB]) {
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const auto p = span(in, b, lane, lanes);
      w[b].zero();
      if (p.in) w[b].load(weight + p.at, kC, false);
    }
  }

  __device__ __forceinline__ void load(const In& in, int64_t i, uint32_t lane, uint32_t lanes, const Mat<const T>& g,
                                       const Mat<const T>& x16, const Mat8& x8, const Mat<const T>& d, const float* rstd) {
    r = rstd[i];
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const auto p = span(in, b, lane, lanes);
      grad[b].zero();
      dsum[b].zero();
      x[b].zero();
      if (!p.in) continue;
      grad[b].template load<true>(g.p + i * g.ld + p.at, kC, false);
      x[b].load(x16, x8, i, p);
      if (d.p) dsum[b].template load<true>(d.p + i * d.ld + p.at, kC, false);
    }
  }

  // the lane's part of the products dn n; kSum: adds grad n to the columns' sums
  template <bool kSum>
  __device__ __forceinline__ float products(const In& in, uint32_t lane, uint32_t lanes, const Block (&weight)[kB],
                                            float (&sums)[kB][kC]) const {
    float dot = 0.0f;
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const auto p = span(in, b, lane, lanes);
      float g[kC], n[kC], w[kC];
      grad[b].widen(g, kC);
      x[b].widen(n, kC, r);
      weight[b].widen(w, kC);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) {
        if (kSum) sums[b][e] += g[e] * n[e];
        dot += p.counts(e) ? g[e] * w[e] * n[e] : 0.0f;
      }
    }
    return dot;
  }

  __device__ __forceinline__ void store(const In& in, int64_t i, uint32_t lane, uint32_t lanes, const Block (&weight)[kB], float mean,
                                        const Mat<T>& dx) const {
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) {
      const auto p = span(in, b, lane, lanes);
      if (!p.in) continue;
      float g[kC], n[kC], w[kC], d[kC];
      grad[b].widen(g, kC);
      x[b].widen(n, kC, r);
      weight[b].widen(w, kC);
      dsum[b].widen(d, kC);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) d[e] += r * (g[e] * w[e] - n[e] * mean);
      store_block<true, true>(dx.p + i * dx.ld + p.at, kC, d);
    }
  }
};

// kShared: rows within a wavefront, which has as many at a time as it has runs of `lanes` lanes for; a workgroup's
// wavefronts meet only at the end, to join their sums.  In us, with that, without it, and with a row to a wavefront:
// 65536 rows of 64 bf16 13.3, 16.5, 32.7; 131072 of 256 50.8, 60.6, 62.1; 32768 of 512 27.5, 39.4 (both).
template <typename T, uint32_t kB, bool kWhole, Kind8 k8, bool kSum, bool kShared>
__global__ __launch_bounds__(kMostWaves * 64) void norm_grad_kernel(In in, Mat<const T> grad, Mat<const T> x, Mat8 x8,
                                                                    const T* weight, Mat<const T> dsum, Mat<T> dx,
                                                                    const float* rstd, float* partial) {
  using R = Row<T, kB, kWhole, k8>;
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t lanes = kShared ? in.lanes : blockDim.x, lane = kShared ? threadIdx.x % lanes : threadIdx.x;
  const uint32_t at_once = kShared ? blockDim.x / lanes : 1, mine = kShared ? threadIdx.x / lanes : 0;
  typename R::Block w[kB];
  R::load_weight(in, lane, lanes, weight, w);
  float sums[kB][kC] = {};
  uint32_t turn = 0;
  for (uint64_t row = uint64_t(blockIdx.x) * at_once + mine; row < in.rows; row += uint64_t(gridDim.x) * at_once, turn = 1 - turn) {
    R now;
    now.load(in, int64_t(row), lane, lanes, grad, x, x8, dsum, rstd);
    compiler_fence();
    const float dot = now.template products<kSum>(in, lane, lanes, w, sums);
    float all;
    if constexpr (kShared) all = lanes_sum(dot, lanes);
    else all = row_sum(dot, blockDim.x / 64, turn);
    now.store(in, int64_t(row), lane, lanes, w, all * in.per_col, dx);
  }
  if (!kSum) return;
  if constexpr (kShared) {  // over the wavefront's rows, then over the wavefronts
    extern __shared__ __attribute__((aligned(16))) float joined[];
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e)
      for (uint32_t d = lanes; d < 64; d *= 2) sums[0][e] += __shfl_xor(sums[0][e], int(d));
    if (blockDim.x > 64) {
      if (threadIdx.x % 64 < lanes) store_sums(joined + (threadIdx.x / 64 * lanes + lane) * kC, sums[0]);
      __syncthreads();
    }
    if (mine) return;
    for (uint32_t v = 1; v < blockDim.x / 64; ++v) {
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) sums[0][e] += joined[(v * lanes + lane) * kC + e];
    }
  }
#pragma unroll
  for (uint32_t b = 0; b < kB; ++b) {
    const auto p = R::span(in, b, lane, lanes);
    if (p.in) store_sums(partial + uint64_t(blockIdx.x) * in.cols + p.at, sums[b]);
  }
}

// Few rows, in one launch: the first workgroups have kFewBlocks blocks of columns and
// all rows, and so the whole of dweight's sums; the others have rows, as many at
// once as their wavefronts hold.  grad and x are read twice, the second time from the caches.
constexpr uint32_t kFewThreads = 1024, kBatch = 2;
constexpr uint32_t kXcds = 8;

template <typename T, uint32_t kFewBlocks, bool kWhole, Kind8 k8>
__device__ __forceinline__ void few_columns(const In& in, uint32_t slab, const Mat<const T>& grad, const Mat<const T>& x,
                                            const Mat8& x8, const float* rstd, float* dweight, uint32_t accumulate) {
  constexpr uint32_t kC = kLaneCols<T>, kWaves = kFewThreads / 64, kFewDown = kFewThreads / kFewBlocks;
  __shared__ float shared[kWaves][kFewBlocks * kC];
  const uint32_t across = threadIdx.x % kFewBlocks, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint64_t left = uint64_t(slab) * kFewBlocks * kC, col = left + across * kC;
  if (left >= in.cols) return;
  const uint32_t width = block_width<kC>(col, in.cols);
  const bool mine = threadIdx.x < kFewBlocks * kC && left + threadIdx.x < in.cols;
  const float before = mine && accumulate ? dweight[left + threadIdx.x] : 0.0f;
  float sum[kC] = {};
  if (width) {
    for (uint32_t i0 = threadIdx.x / kFewBlocks; i0 < in.rows; i0 += kFewDown * kBatch) {
      Raw<T, kC, kWhole> rg[kBatch];
      Input<T, kWhole, k8> rx[kBatch];
      float r[kBatch];
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b) {
        const uint32_t i = i0 + b * kFewDown < in.rows ? i0 + b * kFewDown : i0;
        rg[b].load(grad.p + int64_t(i) * grad.ld + col, width, in.cols < kC);
        rx[b].load(x, x8, i, col, width, in.cols < kC);
        r[b] = rstd[i];
      }
      compiler_fence();
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b) {
        if (i0 + b * kFewDown >= in.rows) break;
        float g[kC], n[kC];
        rg[b].widen(g, width);
        rx[b].widen(n, width, r[b]);
#pragma unroll
        for (uint32_t e = 0; e < kC; ++e) sum[e] += g[e] * n[e];
      }
    }
  }
  // over the wavefront's rows, which lie kFewBlocks lanes apart, then over the wavefronts
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) {
#pragma unroll
    for (uint32_t d = kFewBlocks; d < 64; d *= 2) sum[e] += __shfl_xor(sum[e], int(d));
    if (lane < kFewBlocks) shared[wave][lane * kC + e] = sum[e];
  }
  __syncthreads();
  if (!mine) return;
  float all = 0.0f;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) all += shared[w][threadIdx.x];
  dweight[left + threadIdx.x] = before + all;
}

template <typename T, uint32_t kB, uint32_t kFewBlocks, bool kWhole, Kind8 k8>
__global__ __launch_bounds__(kFewThreads) void norm_grad_few_kernel(In in, uint32_t slabs, uint32_t waves, Mat<const T> grad,
                                                                    Mat<const T> x, Mat8 x8, const T* weight, Mat<const T> dsum,
                                                                    Mat<T> dx, const float* rstd, float* dweight,
                                                                    uint32_t accumulate) {
  constexpr uint32_t kC = kLaneCols<T>;
  if (blockIdx.x < slabs) {  // neighbours, which share lines, on one XCD
    few_columns<T, kFewBlocks, kWhole, k8>(in, blockIdx.x % kXcds * (slabs / kXcds) + blockIdx.x / kXcds, grad, x, x8, rstd, dweight, accumulate);
    return;
  }
  const uint32_t wave = threadIdx.x / 64, group = wave / waves, groups = kFewThreads / 64 / waves;
  const uint32_t lanes = waves * 64, lane = threadIdx.x - group * lanes;
  const uint32_t row = (blockIdx.x - slabs) * groups + group;
  const bool mine = group < groups && row < in.rows;  // the others take part in the barriers
  const int64_t i = mine ? row : 0;
  using R = Row<T, kB, kWhole, k8>;
  typename R::Block w[kB];
  R now;
  if (mine) {
    now.load(in, i, lane, lanes, grad, x, x8, dsum, rstd);
    R::load_weight(in, lane, lanes, weight, w);
  }
  compiler_fence();
  float none[kB][kC], dot = 0.0f;
  if (mine) dot = now.template products<false>(in, lane, lanes, w, none);
  const float mean = row_sum(dot, waves, 0) * in.per_col;
  if (mine) now.store(in, i, lane, lanes, w, mean, dx);
}

// Rows that no workgroup's registers hold, or of less than a block: read twice, the second time from the
// caches, with the columns' sums in the workgroup's row of the workspace.
template <typename T, bool kWhole, Kind8 k8, bool kSum>
__global__ __launch_bounds__(kMostWaves * 64) void norm_grad_long_kernel(In in, Mat<const T> grad, Mat<const T> x, Mat8 x8,
                                                                         const T* weight, Mat<const T> dsum, Mat<T> dx,
                                                                         const float* rstd, float* partial) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t rows = in.rows, cols = in.cols;
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x, turn = 1 - turn) {
    const int64_t i = int64_t(row);
    const float r = rstd[i];
    float dot = 0.0f, mean = 0.0f;
    for (uint32_t pass = 0; pass < 2; ++pass) {
      for (uint64_t col = uint64_t(threadIdx.x) * kC; col < cols; col += uint64_t(blockDim.x) * kC) {
        const uint32_t width = block_width<kC>(col, cols);
        Raw<T, kC, kWhole> rg, rd, rw;
        Input<T, kWhole, k8> rx;
        rd.zero();
        const bool shorter = cols < kC;
        rg.load(grad.p + i * grad.ld + col, width, shorter);
        rx.load(x, x8, i, col, width, shorter);
        rw.load(weight + col, width, shorter);
        if (pass && dsum.p) rd.load(dsum.p + i * dsum.ld + col, width, shorter);
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
      if (pass == 0) mean = row_sum(dot, blockDim.x / 64, turn) * in.per_col;
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
                      : s.lanes    ? norm_grad_kernel<T, 1, kWhole, k8, kSum, true>
                      : s.per == 1 ? norm_grad_kernel<T, 1, kWhole, k8, kSum, false>
                                   : norm_grad_kernel<T, kMostBlocks, kWhole, k8, kSum, false>;
  // without sums a wavefront has its rows and ends
  const uint32_t joined = kSum ? s.joined : 1, at_once = s.lanes ? 64 / s.lanes : 1, threads = s.waves * joined * 64;
  const uint32_t lds = joined > 1 ? joined * s.lanes * kLaneCols<T> * uint32_t(sizeof(float)) : 0;
  auto run = [&](int64_t first, uint32_t rows, uint32_t wgs) -> hipError_t {
    hipLaunchKernelGGL(kernel, dim3(wgs), dim3(threads), lds, stream, In{rows, s.cols, 1.0f / float(s.cols), s.lanes}, cmat<T>(a.grad, first),
                       cmat<T>(a.x, first), mat8(a.x8, first), static_cast<const T*>(a.weight.data), cmat<T>(a.dsum, first),
                       mat<T>(a.dx, first), a.rstd + first, static_cast<float*>(a.workspace));
    return hipGetLastError();
  };
  if (kSum) return run(0, s.rows, s.parts);
  return for_row_groups(a.grad.rows, threads, [&](int64_t first, uint32_t rows) {
    return run(first, rows, (rows + at_once - 1) / at_once);
  });
}

template <typename T, bool kWhole, Kind8 k8>
hipError_t launch_sum(const etc_norm_grad_args& a, hipStream_t stream) {
  const Shape s = shape_of(uint64_t(a.grad.rows), uint64_t(a.grad.cols), kLaneCols<T>);
  if (!a.dweight.data) return launch_rows<T, kWhole, k8, false>(a, s, stream);
  // In place, rows are written while other workgroups would still sum their columns.  (One launch for the columns and
  // one for the rows behind it would give dweight the same bits either way; in us, with that and with sums by rows: 1024 rows
  // of 2048 bf16 12.6, 9.5; of 4096 fp32 24.6, 17.5; 64 of 4096 bf16 6.5, 8.1.)
  const bool in_place = a.dx.data == a.grad.data || a.dx.data == a.x.data;
  if (is_few(s) && !in_place) {
    // blocks of a workgroup that sums columns: two where there are few workgroups and many rows, whose reads then come
    // all at once (1021 x 681 fp32 in 8.5 us, four 9.3, one 11; 1024 x 2048 bf16 10.6, 11.7, 13.9)
    const uint32_t blocks = blocks_per_row(s.cols, kLaneCols<T>), narrow = s.rows > 512 && blocks <= 512 ? 2 : 4;
    const uint32_t slabs = (blocks + narrow - 1) / narrow;
    const uint32_t padded = (slabs + kXcds - 1) / kXcds * kXcds, groups = kFewThreads / 64 / s.waves;
    const auto kernel = s.per != 1    ? norm_grad_few_kernel<T, kMostBlocks, 4, kWhole, k8>
                        : narrow == 2 ? norm_grad_few_kernel<T, 1, 2, kWhole, k8>
                                      : norm_grad_few_kernel<T, 1, 4, kWhole, k8>;
    hipLaunchKernelGGL(kernel, dim3(padded + (s.rows + groups - 1) / groups), dim3(kFewThreads), 0, stream,
                       In{s.rows, s.cols, 1.0f / float(s.cols), 0}, padded, s.waves, cmat<T>(a.grad, 0), cmat<T>(a.x, 0), mat8(a.x8, 0),
                       static_cast<const T*>(a.weight.data), cmat<T>(a.dsum, 0), mat<T>(a.dx, 0), a.rstd,
                       static_cast<float*>(a.dweight.data), uint32_t(a.accumulate != 0));
    return hipGetLastError();
  }
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
