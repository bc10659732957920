// embed_grad.hip -- the gradient of the embedding table, by sorted ids
// (etc_embed_grad).
//
//   dtable[r, :] (+)= scale * sum over i with id_i - row0 = r of drop'(grad[i, :])
//
// Few tokens: one launch.  The first token of each row finds the others in the
// list and sums them.
// Many: the tokens are put in the order (row, token) by sorting tiles and merging
// them.  The ordered list is cut into chunks of equal length, whatever the runs
// of equal rows are, so that a frequent id keeps no wavefront longer than a rare
// one: a wavefront sums one chunk over 512 columns and writes the rows whose
// runs lie inside it.  The parts of a run that crosses chunks go to the
// workspace and are joined afterwards.
// All sums are in 32 bits and in a fixed order.  Ids below the table come first in
// the list and ids above it last, so the cuts lie in the same places of every run
// whichever rows the table holds: a share's gradient has the bits of the whole's.
//
// The sums are HBM bound (a row of grad per token and of dtable per row, and the
// parts); the other launches are a few waits long.  bf16 gradients, MI355X, in us,
// medians of a trace:
//                                            order       sums                    join
//   16384 x 2048 into 50304 rows, added,     4.8 + 4.7   32, 169 MB, 5.2 TB/s    7.1
//     dropout
//   8192 x 4096 into 8000 rows, written      4.8 + 4.6   37, 191 MB, 5.2 TB/s    5.5
//   128 x 256 into 1024 rows, written        4.2 in all (few)
// (an addition of three tensors of this size by one elementwise kernel reaches 5.6 TB/s).
// What was slower: a radix sort (32 us), atomics-free counts of all pairs (1.8 ms),
// runs that end in the next chunk summed by the wavefront they begin in, which saves
// parts but leaves chunks of unequal length (the same to 2 us more), and the rows of no token
// written by the join's launch instead of the sums' (2 to 5 us more).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kWave = 64;
constexpr uint32_t kNone = 0xFFFFFFFFu;  // no row and no key: those are at most 2^31

struct Tokens {
  Ids ids;
  int64_t row0;
  uint32_t rows, n;
  // token i's row of the table, or `rows` for ids outside it
  __device__ __forceinline__ uint32_t row(uint32_t i) const {
    const uint64_t k = uint64_t(ids.at(i)) - uint64_t(row0);
    return k < rows ? uint32_t(k) : rows;
  }
  // What tokens are ordered by: row + 1, with ids below the table before all of
  // its rows and ids above after them.  So a row's tokens have the places that they
  // have in the order of all ids, whichever of the rows the table holds.
  __device__ __forceinline__ uint32_t key(uint32_t i) const {
    const int64_t id = ids.at(i);
    const uint64_t k = uint64_t(id) - uint64_t(row0);
    return id < row0 ? 0 : (k < rows ? uint32_t(k) : rows) + 1;
  }
};

// Of a key: whether it is a row's.
__device__ __forceinline__ bool is_row(uint32_t key, uint32_t rows) { return key - 1 < rows; }

// LDS that the lanes of one wavefront exchange through: its accesses are in
// order, so only the compiler has to be kept from moving them.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---------------------------------------------------------------------------
// Order.  A token's place in a sorted list is the number of tokens before it:
// smaller keys, and equal ones of earlier tokens.  A tile's are found by
// comparing each with all; then, level by level, runs of sorted tokens become
// one, a token's place being its own in its run plus what a binary search finds
// before it in each of the other runs.  No counters, so no order of arrival.  Either
// way a workgroup places 64 tokens, and its 16 wavefronts share what they are
// compared with, so that a launch is a few waits long however many tokens there are.

constexpr uint32_t kPlaceWaves = 16;
constexpr uint32_t kPlaceThreads = kPlaceWaves * kWave;
constexpr uint32_t kTile = kPlaceWaves * kWave;  // a wavefront compares with 64 keys

// The sum over the workgroup's wavefronts of what each counted, in the first of them.
__device__ __forceinline__ uint32_t total_place(uint32_t (&count)[kPlaceWaves][kWave], uint32_t place) {
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  count[wave][lane] = place;
  __syncthreads();
  uint32_t total = 0;
  if (wave == 0)
#pragma unroll
    for (uint32_t w = 0; w < kPlaceWaves; ++w) total += count[w][lane];
  return total;
}

// Tiles of kEach kTile tokens.  Up to 2 kTile tokens are one tile: 2048 x 2048, 17.8 us,
// where two tiles and a merge took 20.1; as runs to merge larger tiles cost 2 us more.
template <uint32_t kEach>
__global__ __launch_bounds__(kPlaceThreads) void tile_kernel(Tokens t, uint32_t* keys, uint32_t* order) {
  constexpr uint32_t kBlocks = kPlaceWaves * kEach;
  __shared__ __attribute__((aligned(16))) uint32_t all[kPlaceWaves][kEach][kWave];
  __shared__ uint32_t count[kPlaceWaves][kWave];
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t mine = blockIdx.x, i = mine * kWave + lane;
  const uint32_t first = mine / kBlocks * kBlocks * kWave, others = mine / kBlocks * kBlocks + wave * kEach;
  const uint32_t key = i < t.n ? t.key(i) : kNone;
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k) {
    const uint32_t j = (others + k) * kWave + lane;
    all[wave][k][lane] = j < t.n ? t.key(j) : kNone;
  }
  wave_sync();
  uint32_t place = 0;
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k) {
    if (others + k != mine) {
      const uint32_t below = key + (others + k < mine);  // equal keys of earlier tokens come before
#pragma unroll
      for (uint32_t e = 0; e < kWave; ++e) place += all[wave][k][e] < below;
    } else {
#pragma unroll
      for (uint32_t e = 0; e < kWave; ++e) place += all[wave][k][e] < key + (e < lane);
    }
  }
  place = total_place(count, place);
  if (wave == 0 && i < t.n) {
    keys[first + place] = key;
    order[first + place] = i;
  }
}

// kEach runs per wavefront become one with those of the other wavefronts.
// kTiles: the runs are tiles, which are staged in LDS.
template <bool kTiles, uint32_t kEach>
__global__ __launch_bounds__(kPlaceThreads) void merge_kernel(uint32_t n, uint32_t length, const uint32_t* keys,
                                                              const uint32_t* order, uint32_t* to_keys,
                                                              uint32_t* to_order) {
  constexpr uint32_t kRuns = kEach * kPlaceWaves;
  __shared__ uint32_t staged[kTiles ? kPlaceWaves : 1][kEach][kTiles ? kTile : 1];
  __shared__ uint32_t count[kPlaceWaves][kWave];
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t from = blockIdx.x * kWave, i = from + lane;  // one run's: lengths are multiples of 64
  const uint32_t run = from / length, group = run / kRuns * kRuns;
  const uint32_t key = i < n ? keys[i] : 0;
  uint32_t first[kEach], size[kEach];
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k) {
    const uint64_t start = uint64_t(group + wave + k * kPlaceWaves) * length;
    first[k] = uint32_t(start < n ? start : 0);
    size[k] = start < n ? min(length, n - uint32_t(start)) : 0;
  }
  if constexpr (kTiles) {
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
      uint32_t v[kTile / kWave];
#pragma unroll
      for (uint32_t e = 0; e < kTile / kWave; ++e) {
        const uint32_t x = e * kWave + lane;
        v[e] = x < size[k] ? keys[first[k] + x] : kNone;
      }
#pragma unroll
      for (uint32_t e = 0; e < kTile / kWave; ++e) staged[wave][k][e * kWave + lane] = v[e];
    }
    wave_sync();
  }
  // how many keys of each run come before, all of its runs' searches side by side
  uint32_t below[kEach], at[kEach] = {};
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k)
    below[k] = key + (group + wave + k * kPlaceWaves < run);  // equal keys of earlier runs come before
  for (uint32_t step = length; step; step /= 2) {
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
      const uint32_t to = at[k] + step;
      const uint32_t* list = kTiles ? staged[wave][k] : keys + first[k];
      if (to <= size[k] && list[to - 1] < below[k]) at[k] = to;
    }
  }
  uint32_t place = 0;
#pragma unroll
  for (uint32_t k = 0; k < kEach; ++k) place += group + wave + k * kPlaceWaves == run ? i - run * length : at[k];
  place = total_place(count, place);
  if (wave == 0 && i < n) {
    const uint32_t to = group * length + place;
    to_keys[to] = key;
    to_order[to] = order[i];
  }
}

// ---------------------------------------------------------------------------
// Sums

constexpr uint32_t kSumThreads = 256;
constexpr uint32_t kSumWaves = kSumThreads / kWave;
constexpr uint32_t kAddBatch = 4, kSetBatch = 8;  // rows in flight per wavefront

struct SumArgs {
  const uint32_t *keys, *order;
  float* parts;      // [chunk][2][cols]: 0 of the run that came in, 1 of the run that goes on
  uint32_t n, rows, cols, accumulate;
  uint32_t chunk, chunks, slabs;
  uint32_t sum_wgs;    // workgroups that sum; the rest write the rows of no token
  uint32_t fill_rows;  // of few tokens: rows per workgroup of these
  float scale;
  Drop drop;
};

// A row of the table that a run ends in: what it holds (kAdd; read early) and the sum.
template <bool kAdd, bool kWhole, uint32_t kC>
__device__ __forceinline__ void finish_row(const SumArgs& a, const Mat<float>& out, uint32_t row, uint64_t col,
                                           uint32_t width, const float (&sum)[kC], const Raw<float, kC, kWhole>& before) {
  float v[kC] = {};
  if (kAdd) before.widen(v, width);
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) v[e] += sum[e] * a.scale;
  store_block<kWhole>(out.p + int64_t(row) * out.ld + col, width, v);
}

template <bool kWhole, uint32_t kC>
__device__ __forceinline__ void read_row(const SumArgs& a, const Mat<float>& out, uint32_t row, uint64_t col,
                                         uint32_t width, Raw<float, kC, kWhole>& before) {
  if (a.accumulate) before.load(out.p + int64_t(row) * out.ld + col, width, a.cols < kC);
  else before.zero();
}

// The first place whose key is at least `key`, found by all lanes of a wavefront together, 64 places at a time.
__device__ __forceinline__ uint32_t lower_bound(const uint32_t* keys, uint32_t n, uint32_t key, uint32_t lane) {
  uint32_t lo = 0, len = n;  // the answer lies in lo .. lo + len
  while (len > 0) {
    const uint32_t step = (len + kWave - 1) / kWave;
    const uint32_t at = lo + (lane + 1) * step - 1;  // the last place of each lane's part
    const bool less = (lane + 1) * step <= len && keys[at] < key;
    const uint32_t full = uint32_t(__popcll(__ballot(less)));  // whole parts below: the first `full` ones
    lo += full * step;
    len -= full * step;
    if (len >= step) len = step - 1;  // the next part's last key is not below
  }
  return lo;
}

__device__ __forceinline__ void zero_row(const SumArgs& a, const Mat<float>& out, uint32_t row, uint32_t lane) {
  constexpr uint32_t kC = kLaneCols<float>;
  const float zero[kC] = {};
  for (uint64_t col = lane * kC; col < a.cols; col += kWave * kC)
    store_block<false>(out.p + int64_t(row) * out.ld + col, block_width<kC>(col, a.cols), zero);
}

// Zeros in the rows of no token, a wavefront per row.
__device__ __forceinline__ void fill_rows(const SumArgs& a, const Mat<float>& out) {
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t waves = (gridDim.x - a.sum_wgs) * kSumWaves;
  for (uint32_t r = (blockIdx.x - a.sum_wgs) * kSumWaves + threadIdx.x / kWave; r < a.rows; r += waves) {
    const uint32_t at = lower_bound(a.keys, a.n, r + 1, lane);
    if (at == a.n || a.keys[at] != r + 1) zero_row(a, out, r, lane);
  }
}

template <typename T, bool kWhole, bool kDrop, bool kAdd>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(SumArgs a, Mat<const T> grad, Mat<float> out) {
  constexpr uint32_t kC = kLaneCols<T>, kBatch = kAdd ? kAddBatch : kSetBatch;
  if (blockIdx.x >= a.sum_wgs) {
    fill_rows(a, out);
    return;
  }
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t job = __builtin_amdgcn_readfirstlane(blockIdx.x * kSumWaves + threadIdx.x / kWave);
  const uint32_t chunk = job / a.slabs;
  if (chunk >= a.chunks) return;
  // the chunk's keys and tokens, one per lane
  const uint32_t lo = chunk * a.chunk, size = min(a.chunk, a.n - lo);
  const uint32_t key = lane < size ? a.keys[lo + lane] : kNone, token = lane < size ? a.order[lo + lane] : 0;
  const uint32_t prev = lo > 0 ? a.keys[lo - 1] : kNone, next = lo + size < a.n ? a.keys[lo + size] : kNone;
  const uint64_t held = __ballot(is_row(key, a.rows));  // consecutive ones: begin .. end
  if (held == 0) return;
  const uint32_t begin = uint32_t(__builtin_ctzll(held)), end = begin + uint32_t(__popcll(held));
  const uint32_t after = __shfl_down(key, 1);
  const uint64_t ends = __ballot(is_row(key, a.rows) && (lane + 1 == size ? next : after) != key);
  // the run that began in an earlier chunk: its end here goes to the parts, not to the table
  uint32_t came = begin == 0 && __builtin_amdgcn_readfirstlane(key) == prev ? (ends ? uint32_t(__builtin_ctzll(ends)) : end) : kNone;

  const uint64_t col = (uint64_t(job - chunk * a.slabs) * kWave + lane) * kC;
  const uint32_t width = block_width<kC>(col, a.cols);
  float* parts = a.parts + uint64_t(chunk) * 2 * a.cols + col;
  float sum[kC] = {};
  // lanes past the columns load block 0, so that the loads are in one piece of code without branches
  const uint64_t from = width ? col : 0;
  const uint32_t span = width ? width : block_width<kC>(0, a.cols);
  for (uint32_t e0 = begin; e0 < end; e0 += kBatch) {
    uint32_t i[kBatch], row[kBatch];
    Raw<T, kC, kWhole> raw[kBatch];
    Raw<float, kC, kWhole> before[kBatch];
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
      const uint32_t e = min(e0 + b, end - 1);
      i[b] = __builtin_amdgcn_readlane(token, e);
      row[b] = __builtin_amdgcn_readlane(key, e) - 1;
      raw[b].template load<true>(grad.p + int64_t(i[b]) * grad.ld + from, span, a.cols < kC);
    }
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b)
      if (kAdd && e0 + b < end && (ends >> (e0 + b) & 1) && e0 + b != came)
        before[b].load(out.p + int64_t(row[b]) * out.ld + from, span, a.cols < kC);
    compiler_fence();
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
      const uint32_t e = e0 + b;
      if (e >= end) break;
      uint32_t bits[kC / 2];
      if (kDrop) a.drop.template bits<kC>(i[b], col, bits);
      float v[kC];
      raw[b].widen(v, width);
      if (kDrop) a.drop.template apply<kC>(bits, v);
#pragma unroll
      for (uint32_t x = 0; x < kC; ++x) sum[x] += v[x];
      if (ends >> e & 1) {
        if (width) {
          if (e == came) store_block<kWhole>(parts, width, sum);
          else finish_row<kAdd>(a, out, row[b], col, width, sum, before[b]);
        }
#pragma unroll
        for (uint32_t x = 0; x < kC; ++x) sum[x] = 0.0f;
      }
    }
  }
  // a run that goes on: part 0 where it fills the chunk and came in, else part 1
  if (!(ends >> (end - 1) & 1) && width) store_block<kWhole>(parts + (came == end ? 0 : a.cols), width, sum);
}

constexpr uint32_t kJoinWaves = 4;
constexpr uint32_t kJoinBatch = 4;  // parts in flight per wavefront

// Joins the parts of the run that begins in this chunk and goes on in the next
// ones: a workgroup per chunk and slab, its wavefronts taking the parts in turn.
template <bool kWhole, uint32_t kC>
__global__ __launch_bounds__(kJoinWaves* kWave) void join_kernel(SumArgs a, Mat<float> out) {
  __shared__ float shared[kJoinWaves][kWave][kC];
  const uint32_t chunk = blockIdx.x / a.slabs, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t lo = chunk * a.chunk, hi = lo + a.chunk;  // not the last chunk
  // the keys that decide, in one wait: around both ends, and the first ones of the next 64 chunks
  const uint32_t run = a.keys[hi - 1], prev = lo > 0 ? a.keys[lo - 1] : kNone, head = a.keys[lo];
  uint32_t next = chunk + 1 + lane;
  uint32_t key = next < a.chunks ? a.keys[next * a.chunk] : kNone;
  if (!is_row(run, a.rows) || __builtin_amdgcn_readfirstlane(key) != run) return;
  if (head == run && prev == run) return;  // it began before this chunk
  // the chunks that the run reaches: those whose first key is the run's
  uint32_t parts = 0;
  for (;;) {
    const uint32_t more = uint32_t(__popcll(__ballot(key == run)));
    parts += more;
    if (more < kWave) break;
    next += kWave;
    key = next < a.chunks ? a.keys[next * a.chunk] : kNone;
  }
  const uint64_t col = (uint64_t(blockIdx.x - chunk * a.slabs) * kWave + lane) * kC;
  const uint32_t width = block_width<kC>(col, a.cols);
  float sum[kC] = {};
  Raw<float, kC, kWhole> before;
  before.zero();
  if (width) {
    if (wave == 0) read_row(a, out, run - 1, col, width, before);
    // part 0 is this chunk's own
    for (uint32_t k0 = wave; k0 <= parts; k0 += kJoinWaves * kJoinBatch) {
      Raw<float, kC, kWhole> part[kJoinBatch];
#pragma unroll
      for (uint32_t b = 0; b < kJoinBatch; ++b) {
        const uint32_t k = min(k0 + b * kJoinWaves, parts);
        part[b].load(a.parts + (uint64_t(chunk + k) * 2 + (k == 0)) * a.cols + col, width, a.cols < kC);
      }
      compiler_fence();
#pragma unroll
      for (uint32_t b = 0; b < kJoinBatch; ++b) {
        if (k0 + b * kJoinWaves > parts) break;
        float v[kC];
        part[b].widen(v, width);
#pragma unroll
        for (uint32_t e = 0; e < kC; ++e) sum[e] += v[e];
      }
    }
  }
#pragma unroll
  for (uint32_t e = 0; e < kC; ++e) shared[wave][lane][e] = sum[e];
  __syncthreads();
  if (wave != 0 || !width) return;
#pragma unroll
  for (uint32_t w = 1; w < kJoinWaves; ++w)
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) sum[e] += shared[w][lane][e];
  finish_row<true>(a, out, run - 1, col, width, sum, before);
}

// ---------------------------------------------------------------------------
// Few tokens, in one launch: a workgroup per token and slab, whose lanes look at
// all tokens' keys, 64 tokens to a word of a mask.  The first token of a row
// lists all of the row's and adds them up, its wavefronts a batch at a time in
// turn.  Further workgroups write the rows of no token.

constexpr uint32_t kFewMost = 512;
constexpr uint32_t kFewEach = kFewMost / kSumThreads;  // tokens per lane
constexpr uint32_t kFewBatch = 2;                      // rows in flight per wavefront: most rows have one or two tokens
constexpr uint32_t kWords = kFewMost / kWave;
constexpr uint32_t kFillMost = 16;                     // rows that a workgroup looks for

template <typename T, bool kWhole, bool kDrop>
__global__ __launch_bounds__(kSumThreads) void few_kernel(Tokens t, SumArgs a, Mat<const T> grad, Mat<float> out) {
  constexpr uint32_t kC = kLaneCols<T>;
  __shared__ uint64_t masks[kWords];
  __shared__ uint32_t list[kFewMost];
  __shared__ float shared[kSumWaves][kWave][kC];
  __shared__ uint32_t seen[kFillMost];
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t rows[kFewEach];
#pragma unroll
  for (uint32_t p = 0; p < kFewEach; ++p) {
    const uint32_t i = p * kSumThreads + threadIdx.x;
    rows[p] = i < t.n ? t.row(i) : kNone;
  }
  if (blockIdx.x >= a.sum_wgs) {
    for (uint64_t first = uint64_t(blockIdx.x - a.sum_wgs) * a.fill_rows; first < a.rows;
         first += uint64_t(gridDim.x - a.sum_wgs) * a.fill_rows) {
      if (threadIdx.x < kFillMost) seen[threadIdx.x] = 0;
      __syncthreads();
#pragma unroll
      for (uint32_t p = 0; p < kFewEach; ++p)
        if (rows[p] < a.rows && rows[p] >= first && rows[p] - first < a.fill_rows) seen[rows[p] - first] = 1;
      __syncthreads();
      for (uint32_t r = wave; r < a.fill_rows && first + r < a.rows; r += kSumWaves)
        if (!seen[r]) zero_row(a, out, uint32_t(first) + r, lane);
      __syncthreads();
    }
    return;
  }
  const uint32_t mine = blockIdx.x / a.slabs, row = t.row(mine);
  if (row >= a.rows) return;
#pragma unroll
  for (uint32_t p = 0; p < kFewEach; ++p) {
    const uint64_t same = __ballot(rows[p] == row);
    if (lane == 0) masks[p * kSumWaves + wave] = same;
  }
  __syncthreads();
  // each of this lane's tokens has the tokens of its word and those before it in the list
  uint32_t total = 0, before[kFewEach];
#pragma unroll
  for (uint32_t w = 0; w < kWords; ++w) {
    const uint64_t m = masks[w];
    const uint64_t earlier = mine >= (w + 1) * kWave ? ~uint64_t(0) : mine > w * kWave ? (uint64_t(1) << (mine - w * kWave)) - 1 : 0;
    if (m & earlier) return;  // an earlier token's workgroup does it; the same for the whole workgroup
    if (w % kSumWaves == wave) before[w / kSumWaves] = total + uint32_t(__popcll(m & ((uint64_t(1) << lane) - 1)));
    total += uint32_t(__popcll(m));
  }
#pragma unroll
  for (uint32_t p = 0; p < kFewEach; ++p)
    if (rows[p] == row) list[before[p]] = p * kSumThreads + threadIdx.x;
  __syncthreads();
  const uint64_t col = (uint64_t(blockIdx.x - mine * a.slabs) * kWave + lane) * kC;
  const uint32_t width = block_width<kC>(col, a.cols);
  Raw<float, kC, kWhole> held;
  held.zero();
  if (width && wave == 0) read_row(a, out, row, col, width, held);
  float sum[kC] = {};
  for (uint32_t e0 = wave * kFewBatch; e0 < total; e0 += kSumWaves * kFewBatch) {
    // all loads, then all of the arithmetic without branches, so that the rows' chains of products overlap
    Raw<T, kC, kWhole> raw[kFewBatch];
    uint32_t bits[kFewBatch][kC / 2];
#pragma unroll
    for (uint32_t b = 0; b < kFewBatch; ++b) {
      const uint32_t i = __builtin_amdgcn_readfirstlane(list[min(e0 + b, total - 1)]);
      if (width) raw[b].template load<true>(grad.p + int64_t(i) * grad.ld + col, width, a.cols < kC);
      if (kDrop) a.drop.template bits<kC>(i, col, bits[b]);
    }
#pragma unroll
    for (uint32_t b = 0; b < kFewBatch; ++b) {
      float v[kC];
      raw[b].widen(v, width);
      if (kDrop) a.drop.template apply<kC>(bits[b], v);
#pragma unroll
      for (uint32_t x = 0; x < kC; ++x) sum[x] += e0 + b < total ? v[x] : 0.0f;
    }
  }
  if (total > kFewBatch) {  // other wavefronts have parts
#pragma unroll
    for (uint32_t x = 0; x < kC; ++x) shared[wave][lane][x] = sum[x];
    __syncthreads();
    if (wave == 0)
#pragma unroll
      for (uint32_t w = 1; w < kSumWaves; ++w)
#pragma unroll
        for (uint32_t x = 0; x < kC; ++x) sum[x] += shared[w][lane][x];
  }
  if (wave == 0 && width) finish_row<true>(a, out, row, col, width, sum, held);
}

// ---------------------------------------------------------------------------

// Few tokens or many, at most so many tokens and workgroups that sum: few waits
// less (one launch, where many take three or four, at 2.3 us of the host's time
// each) but leaves a frequent id to four wavefronts, whose arithmetic it then
// waits for.  MI355X, graph replays, in us, few / many, accumulated, dropout:
//   columns   ids log-uniform                     all ids alike
//      256    256: 5.1 / 10.2   512: 7.4 / 10.5    256: 21 / 11.6   512: 39 / 14.6
//     2048    256: 4.9 / 10.2   512: 6.5 / 10.6    256: 21 / 12.1   512: 39 / 15.1
//     8192    128: 6.9 / 10.2   512: 22 / 13.4     128: 11.8 / 10.5
// (half of 512 ids alike: 21 to 22).  The choice is made on the host, which does not
// see the ids, so a batch that is padded with an id of the table pays for it.
constexpr uint64_t kFewJobs = 2048;

// Slabs of a row: a wavefront's 64 blocks of `block` columns.
uint64_t slabs_of(uint64_t cols, uint32_t block) { return (cols + kWave * block - 1) / (kWave * block); }

bool is_few(uint64_t n, uint64_t slabs) { return n <= kFewMost && n * slabs <= kFewJobs; }

// Tokens per chunk: 4 to 64 (one per lane), so that there are at most kJobs
// wavefronts, and kChunks chunks, for each of which the join has a workgroup per
// slab.  16384 x 2048, MI355X, in us, with 2048 / 4096 / 6144 jobs: 51.5 / 48.2 /
// 52.5; 16384 x 256 with at most 4096 / 2048 / 1024 chunks: 32.7 / 26.1 / 23.4.
constexpr uint64_t kJobs = 4096, kChunks = 1024, kChunkLeast = 4, kChunkMost = kWave;

uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

uint32_t chunk_of(uint64_t n, uint64_t slabs) {
  return uint32_t(std::min(kChunkMost, std::max({kChunkLeast, up(n * slabs, kJobs), up(n, kChunks)})));
}

// Columns of parts, at most, over all chunks: n / kChunkLeast of them, or where
// chunks are longer kJobs / slabs, or where those would pass kChunkMost tokens
// n / kChunkMost.  It grows with n and cols, so a workspace serves smaller calls.
uint64_t part_cols(uint64_t n, uint64_t cols) {
  return std::min(up(n, kChunkLeast) * cols, std::max(kJobs * kWave * kLaneCols<bf16> + cols, up(n, kChunkMost) * cols));
}

hipError_t sort_tokens(const Tokens& t, char* work, const EmbedGradSizes& w, const uint32_t** keys,
                       const uint32_t** order, hipStream_t stream) {
  auto at = [&](uint64_t byte) { return reinterpret_cast<uint32_t*>(work + byte); };
  const dim3 wgs((t.n + kWave - 1) / kWave), block(kPlaceThreads);
  const bool one = t.n <= 2 * kTile;
  hipLaunchKernelGGL(one && t.n > kTile ? tile_kernel<2> : tile_kernel<1>, wgs, block, 0, stream, t, at(w.keys[0]), at(w.order[0]));
  uint32_t in = 0;  // the pair of lists that holds the runs
  for (uint64_t length = kTile, runs = kPlaceWaves; !one && length < t.n; length *= runs, runs = 4 * kPlaceWaves) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto merge = length == kTile ? merge_kernel<true, 1> : merge_kernel<false, 4>;
    hipLaunchKernelGGL(merge, wgs, block, 0, stream, t.n, uint32_t(length), at(w.keys[in]), at(w.order[in]),
                       at(w.keys[in ^ 1]), at(w.order[in ^ 1]));
    in ^= 1;
  }
  *keys = at(w.keys[in]);
  *order = at(w.order[in]);
  return hipGetLastError();
}

template <typename T, bool kAdd>
auto sum_kernel_for(bool whole, bool drop) {
  return drop ? whole ? sum_kernel<T, true, true, kAdd> : sum_kernel<T, false, true, kAdd>
              : whole ? sum_kernel<T, true, false, kAdd> : sum_kernel<T, false, false, kAdd>;
}

template <typename T>
hipError_t launch(const etc_embed_grad_args& x, const Drop& drop, hipStream_t stream) {
  const uint32_t n = uint32_t(x.tokens.count), rows = uint32_t(x.dtable.rows), cols = uint32_t(x.dtable.cols);
  const EmbedGradSizes w = embed_grad_sizes(n, rows, cols);
  char* work = static_cast<char*>(x.workspace);
  const Tokens t{Ids{x.tokens.data, x.tokens.dtype == ETC_IDS_I64}, x.row0, rows, n};
  const Mat<const T> grad{static_cast<const T*>(x.grad.data), x.grad.ld};
  const Mat<float> out{static_cast<float*>(x.dtable.data), x.dtable.ld};
  const dim3 block(kSumThreads);
  const bool whole = whole_blocks(cols, kLaneCols<T>);
  SumArgs a{};
  a.n = n;
  a.rows = rows;
  a.cols = cols;
  a.accumulate = x.accumulate != 0;
  a.slabs = uint32_t(slabs_of(cols, kLaneCols<T>));
  a.scale = float(x.scale);
  a.drop = drop;
  if (is_few(n, a.slabs)) {
    a.sum_wgs = n * a.slabs;
    a.fill_rows = a.slabs == 1 ? kFillMost : kSumWaves;
    const dim3 wgs(a.sum_wgs + (a.accumulate ? 0 : std::min((rows + a.fill_rows - 1) / a.fill_rows, 1u << 20)));
    const auto few = drop.limit ? whole ? few_kernel<T, true, true> : few_kernel<T, false, true>
                                : whole ? few_kernel<T, true, false> : few_kernel<T, false, false>;
    hipLaunchKernelGGL(few, wgs, block, 0, stream, t, a, grad, out);
    return hipGetLastError();
  }
  const hipError_t e = sort_tokens(t, work, w, &a.keys, &a.order, stream);
  if (e != hipSuccess) return e;
  a.parts = reinterpret_cast<float*>(work + w.parts);
  a.chunk = chunk_of(n, a.slabs);
  a.chunks = (n + a.chunk - 1) / a.chunk;
  a.sum_wgs = uint32_t((uint64_t(a.chunks) * a.slabs + kSumWaves - 1) / kSumWaves);
  const dim3 wgs(a.sum_wgs + (a.accumulate ? 0 : std::min((rows + kSumWaves - 1) / kSumWaves, 1u << 20)));
  const auto sum = a.accumulate ? sum_kernel_for<T, true>(whole, drop.limit) : sum_kernel_for<T, false>(whole, drop.limit);
  hipLaunchKernelGGL(sum, wgs, block, 0, stream, a, grad, out);
  if (a.chunks == 1) return hipGetLastError();  // nothing crosses
  const auto join = whole ? join_kernel<true, kLaneCols<T>> : join_kernel<false, kLaneCols<T>>;
  hipLaunchKernelGGL(join, dim3((a.chunks - 1) * a.slabs), dim3(kJoinWaves * kWave), 0, stream, a, out);
  return hipGetLastError();
}

}  // namespace

EmbedGradSizes embed_grad_sizes(uint64_t n, uint64_t, uint64_t cols) {
  EmbedGradSizes w{};
  auto take = [&](uint64_t bytes) {
    const uint64_t at = w.total;
    w.total += (bytes + 255) / 256 * 256;
    return at;
  };
  for (int k = 0; k < 2; ++k) {
    w.keys[k] = take(4 * n);
    w.order[k] = take(4 * n);
  }
  w.parts = take(part_cols(n, cols) * 2 * sizeof(float));
  return w;
}

bool embed_grad_fits(uint64_t n, uint64_t cols) {
  constexpr uint64_t lanes = uint64_t(1) << 31;  // of a launch
  // ordering: a workgroup per 64 tokens; sums: one per chunk (or token) and slab in the largest launch
  const uint64_t slabs = slabs_of(cols, kLaneCols<float>), jobs = (is_few(n, slabs) ? n : up(n, chunk_of(n, slabs))) * slabs;
  return up(n, kWave) * kPlaceThreads <= lanes && jobs * kSumThreads <= lanes;
}

hipError_t launch_embed_grad(const etc_embed_grad_args& a, const Drop& drop, hipStream_t stream) {
  return a.grad.dtype == ETC_DTYPE_F32 ? launch<float>(a, drop, stream) : launch<bf16>(a, drop, stream);
}

}  // namespace etc
