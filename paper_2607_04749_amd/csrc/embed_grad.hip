// embed_grad.hip -- the gradient of the embedding table, by sorted ids
// (etc_embed_grad).
//
//   dtable[r, :] (+)= scale * sum over i with id_i - row0 = r of drop'(grad[i, :])
//
// First each token's place in the order (row, token) is counted, then the
// tokens of each row are summed in that order, in 32 bits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kThreads = 256;

// A token's key: its row of the table, or `rows` for ids outside it, which sort last.
__device__ __forceinline__ uint32_t key_of(const Ids& ids, int64_t row0, uint32_t rows, uint32_t i) {
  const uint64_t k = uint64_t(ids.at(i)) - uint64_t(row0);
  return k < rows ? uint32_t(k) : rows;
}

// A token's place is the number of tokens that come before it: smaller keys, and equal ones of earlier tokens.
__global__ __launch_bounds__(kThreads) void rank_kernel(Ids ids, int64_t row0, uint32_t rows, uint32_t n,
                                                        uint32_t* keys, uint32_t* order) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  const uint32_t mine = i < n ? key_of(ids, row0, rows, i) : 0;
  uint32_t place = 0;
  for (uint32_t j = 0; j < n; ++j) {
    const uint32_t k = key_of(ids, row0, rows, j);
    place += k < mine || (k == mine && j < i);
  }
  if (i < n) {
    keys[place] = mine;
    order[place] = i;
  }
}

// The first place whose key is at least `key`.
__device__ __forceinline__ uint32_t lower_bound(const uint32_t* keys, uint32_t n, uint32_t key) {
  uint32_t lo = 0, hi = n;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

struct SumArgs {
  const uint32_t *keys, *order;
  uint32_t n, rows, cols, accumulate;
  float scale;
  Drop drop;
};

template <typename T, bool kDrop>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a, Mat<const T> grad, Mat<float> out) {
  const uint64_t col = (uint64_t(blockIdx.y) * kThreads + threadIdx.x) * kBlockCols;
  if (col >= a.cols) return;
  const uint32_t width = uint32_t(a.cols - col < kBlockCols ? a.cols - col : kBlockCols);
  for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const uint32_t lo = lower_bound(a.keys, a.n, r), hi = lower_bound(a.keys, a.n, r + 1);
    if (lo == hi && a.accumulate) continue;
    float sum[8] = {};
    for (uint32_t at = lo; at < hi; ++at) {
      const uint32_t i = a.order[at];
      float v[8];
      load8(grad.p + int64_t(i) * grad.ld + col, width, v);
      if (kDrop) a.drop.apply(i, uint32_t(col / kBlockCols), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
    float* to = out.p + int64_t(r) * out.ld + col;
    float before[8] = {};
    if (a.accumulate) load8(to, width, before);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = before[e] + sum[e] * a.scale;
    store8(to, width, sum);
  }
}

template <typename T>
hipError_t launch(const etc_embed_grad_args& x, const Drop& drop, hipStream_t stream) {
  const uint32_t n = uint32_t(x.tokens.count), rows = uint32_t(x.dtable.rows);
  const EmbedGradSizes w = embed_grad_sizes(n, rows, uint64_t(x.dtable.cols));
  char* work = static_cast<char*>(x.workspace);
  uint32_t *keys = reinterpret_cast<uint32_t*>(work + w.keys), *order = reinterpret_cast<uint32_t*>(work + w.order);
  if (n) {
    hipLaunchKernelGGL(rank_kernel, dim3((n + kThreads - 1) / kThreads), dim3(kThreads), 0, stream,
                       Ids{x.tokens.data, x.tokens.dtype == ETC_IDS_I64}, x.row0, rows, n, keys, order);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const SumArgs a{keys, order, n, rows, uint32_t(x.dtable.cols), uint32_t(x.accumulate != 0), float(x.scale), drop};
  const Mat<const T> grad{static_cast<const T*>(x.grad.data), x.grad.ld};
  const Mat<float> out{static_cast<float*>(x.dtable.data), x.dtable.ld};
  const dim3 wgs(std::min(rows, 65536u), (blocks_per_row(x.dtable.cols) + kThreads - 1) / kThreads), block(kThreads);
  if (drop.limit) hipLaunchKernelGGL((sum_kernel<T, true>), wgs, block, 0, stream, a, grad, out);
  else hipLaunchKernelGGL((sum_kernel<T, false>), wgs, block, 0, stream, a, grad, out);
  return hipGetLastError();
}

}  // namespace

EmbedGradSizes embed_grad_sizes(uint64_t ntokens, uint64_t, uint64_t) {
  auto up = [](uint64_t v) { return (v + 255) / 256 * 256; };
  EmbedGradSizes w{};
  w.keys = 0;
  w.order = up(4 * ntokens);
  w.total = w.order + up(4 * ntokens);
  return w;
}

hipError_t launch_embed_grad(const etc_embed_grad_args& a, const Drop& drop, hipStream_t stream) {
  return a.grad.dtype == ETC_DTYPE_F32 ? launch<float>(a, drop, stream) : launch<bf16>(a, drop, stream);
}

}  // namespace etc
