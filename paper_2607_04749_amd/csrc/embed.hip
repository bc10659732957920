// embed.hip -- the lookup of a rank's share of the vocabulary, with scaling,
// positions and dropout in one pass (etc_embed).
//
//   out[i, :] = drop(scale * table[id_i - row0, :] + pos_table[position_i, :])
//
// HBM bound: it reads the rows that occur and writes one row per token.  A
// lane moves one or two blocks of columns; consecutive lanes and wavefronts follow
// the output, so that it is written as one front, without staying in the caches
// that hold the rows and positions which tokens share.  bf16, MI355X, medians of a trace:
//   8192 x 8192, 227 tokens inside the     21.3 us, 138 MB at the least (6.5 TB/s); 23.2 in graph
//     4000 rows                            replays with the 4000 most frequent ids, most of them inside
//   16384 x 2048 of 50304 rows with 2048   21.4 us: 49 MB read and 67 MB written in
//     positions and dropout                HBM, 201 MB through L2, and about 16 us
//                                          of vector instructions for the mask
//   1 x 4096                               1.8 us: one wait for the id, one for the row
#include <hip/hip_runtime.h>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint64_t kManyBlocks = uint64_t(1) << 20;  // more lanes than the GPU holds at once

template <typename T>
struct EmbedArgs {
  Mat<const T> table, pos;  // pos.p NULL: no positions
  Ids tokens, positions;
  int64_t row0;
  uint64_t rows, pos_rows;
  float scale;
  Drop drop;
  BlockGrid grid;
};

template <typename T, typename O, bool kWhole, bool kDrop, uint32_t kN>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs<T> a, Mat<O> out) {
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  if (at >= a.grid.n) return;
  constexpr uint32_t kC = kLaneCols<O>;
  uint32_t group, block;
  a.grid.place(at, &group, &block);
  const uint64_t col = uint64_t(block) * kC;
  const uint32_t width = block_width<kC>(col, a.grid.cols), i0 = group * kN, last = a.grid.rows - 1;
  const bool shorter = a.grid.cols < kC;
  uint64_t k[kN], q[kN] = {};
#pragma unroll
  for (uint32_t r = 0; r < kN; ++r) {
    const uint32_t i = kN == 1 ? i0 : min(i0 + r, last);
    k[r] = uint64_t(a.tokens.at(i)) - uint64_t(a.row0);  // unsigned: an id below row0 becomes a large row
    if (a.pos.p) q[r] = uint64_t(a.positions.at(i));
  }
  Raw<T, kC, kWhole> word[kN], place[kN];
#pragma unroll
  for (uint32_t r = 0; r < kN; ++r) {
    word[r].zero();
    place[r].zero();
    if (k[r] < a.rows) word[r].load(a.table.p + int64_t(k[r]) * a.table.ld + col, width, shorter);
    if (q[r] < a.pos_rows) place[r].load(a.pos.p + int64_t(q[r]) * a.pos.ld + col, width, shorter);
  }
  compiler_fence();
#pragma unroll
  for (uint32_t r = 0; r < kN; ++r) {
    const uint32_t i = i0 + r;
    if (kN > 1 && i > last) break;
    uint32_t bits[kC / 2];
    if (kDrop) a.drop.template bits<kC>(i, col, bits);  // while the loads are on their way
    float v[kC], w[kC];
    word[r].widen(v, width);
    place[r].widen(w, width);
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) v[e] = v[e] * a.scale + w[e];
    if (kDrop) a.drop.template apply<kC>(bits, v);
    compiler_fence();
    store_block<kWhole, true>(out.p + int64_t(i) * out.ld + col, width, v);
  }
}

template <typename T, typename O, bool kWhole>
auto kernel_for(bool drop, bool two) {
  return two ? embed_kernel<T, O, kWhole, true, 2> : drop ? embed_kernel<T, O, kWhole, true, 1> : embed_kernel<T, O, kWhole, false, 1>;
}

template <typename T, typename O>
hipError_t launch(const etc_embed_args& x, const Drop& drop, hipStream_t stream) {
  EmbedArgs<T> a{};
  a.table = {static_cast<const T*>(x.table.data), x.table.ld};
  a.pos = {static_cast<const T*>(x.pos_table.data), x.pos_table.ld};
  a.row0 = x.row0;
  a.rows = uint64_t(x.table.rows);
  a.pos_rows = x.pos_table.data ? uint64_t(x.pos_table.rows) : 0;
  a.scale = float(x.scale);
  // Two rows per lane where dropout's arithmetic can fill the wait for the
  // second row's loads: 16384 x 2048 with positions and dropout 20.5 us, with one
  // row 22.4; 8192 x 8192 without dropout 22.5 us, with one row 20.8.
  const bool two = drop.limit && uint64_t(x.out.rows) * blocks_per_row(x.out.cols, kLaneCols<O>) >= kManyBlocks;
  const auto kernel = whole_blocks(x.out.cols, kLaneCols<O>) ? kernel_for<T, O, true>(drop.limit, two)
                                                             : kernel_for<T, O, false>(drop.limit, two);
  return for_row_runs(x.out.rows, x.out.cols, kLaneCols<O>, two ? 2 : 1, [&](int64_t first, const BlockGrid& grid) -> hipError_t {
    auto ids = [&](const etc_ids& v) {
      const bool wide = v.dtype == ETC_IDS_I64;
      return Ids{v.data ? static_cast<const char*>(v.data) + first * (wide ? 8 : 4) : nullptr, wide};
    };
    a.tokens = ids(x.tokens);
    a.positions = ids(x.positions);
    a.drop = drop;
    a.drop.row0 += uint64_t(first);
    a.grid = grid;
    const Mat<O> out{static_cast<O*>(x.out.data) + first * x.out.ld, x.out.ld};
    const dim3 wgs((grid.n + kThreads - 1) / kThreads), block(kThreads);
    hipLaunchKernelGGL(kernel, wgs, block, 0, stream, a, out);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_embed(const etc_embed_args& a, const Drop& drop, hipStream_t stream) {
  const bool t32 = a.table.dtype == ETC_DTYPE_F32, o32 = a.out.dtype == ETC_DTYPE_F32;
  if (t32) return o32 ? launch<float, float>(a, drop, stream) : launch<float, bf16>(a, drop, stream);
  return o32 ? launch<bf16, float>(a, drop, stream) : launch<bf16, bf16>(a, drop, stream);
}

}  // namespace etc
