// embed_grad.hip -- the gradient of the embedding table, by sorted ids
// (etc_embed_grad).
//
//   dtable[r, :] (+)= scale * sum over i with id_i - row0 = r of drop'(grad[i, :])
//
// The tokens are put in the order (row, token): few by counting who comes
// before whom, many by a radix sort.  The ordered list is then cut into chunks
// of equal length, whatever the runs of equal rows are, so that a frequent id
// keeps no wavefront longer than a rare one: a wavefront sums one chunk over
// 512 columns and writes the rows whose runs lie inside it.  The parts of a
// run that crosses chunks go to the workspace and are joined afterwards.  All
// sums are in 32 bits and in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kWave = 64;
constexpr uint32_t kNone = 0xFFFFFFFFu;  // no key: keys are at most 2^31 - 1

// A token's key: its row of the table, or `rows` for ids outside it, which sort last.
__device__ __forceinline__ uint32_t key_of(const Ids& ids, int64_t row0, uint32_t rows, uint32_t i) {
  const uint64_t k = uint64_t(ids.at(i)) - uint64_t(row0);
  return k < rows ? uint32_t(k) : rows;
}

struct Tokens {
  Ids ids;
  int64_t row0;
  uint32_t rows, n;
  __device__ __forceinline__ uint32_t key(uint32_t i) const { return key_of(ids, row0, rows, i); }
};

// LDS that the lanes of one wavefront exchange through: its accesses are in
// order, so only the compiler has to be kept from moving them.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---------------------------------------------------------------------------
// Order, few tokens: a token's place is the number of tokens before it, smaller
// keys and equal ones of earlier tokens.  A workgroup places 64 tokens; its 16
// wavefronts share the keys that they are compared with, 64 at a time.

constexpr uint32_t kRankWaves = 16;

__global__ __launch_bounds__(kRankWaves* kWave) void rank_kernel(Tokens t, uint32_t* keys, uint32_t* order) {
  __shared__ __attribute__((aligned(16))) uint32_t other[kRankWaves][kWave];
  __shared__ uint32_t count[kRankWaves][kWave];
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, mine = blockIdx.x;
  const uint32_t i = mine * kWave + lane, blocks = (t.n + kWave - 1) / kWave;
  const uint32_t key = i < t.n ? t.key(i) : 0;
  uint32_t place = 0;
  for (uint32_t b = wave; b < blocks; b += kRankWaves) {
    const uint32_t j = b * kWave + lane;
    other[wave][lane] = j < t.n ? t.key(j) : kNone;
    wave_sync();
    const uint32_t below = key + (b < mine);  // equal keys of earlier blocks come before
    if (b != mine) {
#pragma unroll
      for (uint32_t e = 0; e < kWave; ++e) place += other[wave][e] < below;
    } else {
#pragma unroll
      for (uint32_t e = 0; e < kWave; ++e) place += other[wave][e] < key + (e < lane);
    }
    wave_sync();
  }
  count[wave][lane] = place;
  __syncthreads();
  if (wave == 0 && i < t.n) {
    place = 0;
#pragma unroll
    for (uint32_t w = 0; w < kRankWaves; ++w) place += count[w][lane];
    keys[place] = key;
    order[place] = i;
  }
}

// ---------------------------------------------------------------------------
// Order, many tokens: a radix sort from the low digits up, each pass stable.
// A pass counts the digits of every tile (one workgroup each), and then every
// tile moves its keys: to the keys of smaller digits, and of its own digit in
// earlier tiles, it adds the rank inside the tile.

constexpr uint32_t kSortThreads = 256;
constexpr uint32_t kSortWaves = kSortThreads / kWave;
constexpr uint32_t kMaxDigitBits = 9;
constexpr uint32_t kMaxTiles = 64;  // every tile sums the counts of all

struct SortPass {
  uint32_t tile;   // keys per tile, a multiple of kSortThreads
  uint32_t tiles;  // at most kMaxTiles
  uint32_t shift, bits;
  const uint32_t *keys, *order;  // keys NULL: the first pass, from the ids
  __device__ __forceinline__ uint32_t digit(uint32_t key) const { return (key >> shift) & ((1u << bits) - 1); }
};

__global__ __launch_bounds__(kSortThreads) void digit_kernel(Tokens t, SortPass p, uint32_t* counts) {
  __shared__ uint32_t count[1 << kMaxDigitBits];
  const uint32_t bins = 1u << p.bits;
  for (uint32_t d = threadIdx.x; d < bins; d += kSortThreads) count[d] = 0;
  __syncthreads();
  const uint32_t end = min(t.n, (blockIdx.x + 1) * p.tile);
  for (uint32_t i = blockIdx.x * p.tile + threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&count[p.digit(p.keys ? p.keys[i] : t.key(i))], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < bins; d += kSortThreads) counts[blockIdx.x * bins + d] = count[d];
}

__global__ __launch_bounds__(kSortThreads) void move_kernel(Tokens t, SortPass p, const uint32_t* counts,
                                                            uint32_t* keys, uint32_t* order) {
  __shared__ uint32_t at[kSortWaves][1 << kMaxDigitBits];  // where each wavefront's next key of a digit goes
  __shared__ uint32_t sums[kSortWaves];
  const uint32_t bins = 1u << p.bits, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  for (uint32_t d = threadIdx.x; d < bins; d += kSortThreads)
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) at[w][d] = 0;
  __syncthreads();
  // each wavefront has a quarter of the tile, so earlier wavefronts' keys come first
  const uint32_t quarter = p.tile / kSortWaves, first = blockIdx.x * p.tile + wave * quarter;
  const uint32_t end = min(t.n, first + quarter);
  for (uint32_t i = first + lane; i < end; i += kWave)
    atomicAdd(&at[wave][p.digit(p.keys ? p.keys[i] : t.key(i))], 1u);
  __syncthreads();
  // starts: digits in order (two per thread at most), then tiles, then wavefronts
  uint32_t total[2] = {}, before[2] = {};
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h) {
    const uint32_t d = threadIdx.x * 2 + h;
    if (d < bins)
      for (uint32_t b = 0; b < p.tiles; ++b) {
        const uint32_t c = counts[b * bins + d];
        total[h] += c;
        before[h] += b < blockIdx.x ? c : 0;
      }
  }
  uint32_t scan = total[0] + total[1];
#pragma unroll
  for (uint32_t step = 1; step < kWave; step *= 2) {
    const uint32_t v = __shfl_up(scan, step);
    if (lane >= step) scan += v;
  }
  if (lane == kWave - 1) sums[wave] = scan;
  __syncthreads();
  uint32_t base = scan - total[0] - total[1];
  for (uint32_t w = 0; w < wave; ++w) base += sums[w];
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h) {
    const uint32_t d = threadIdx.x * 2 + h;
    if (d < bins) {
      uint32_t to = base + before[h];
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) {
        const uint32_t c = at[w][d];
        at[w][d] = to;
        to += c;
      }
    }
    base += total[h];
  }
  __syncthreads();
  for (uint32_t i0 = first; i0 < end; i0 += kWave) {  // the same for all lanes of a wavefront
    const uint32_t i = i0 + lane;
    const bool has = i < end;
    const uint32_t key = has ? (p.keys ? p.keys[i] : t.key(i)) : 0, d = p.digit(key);
    // the lanes of the same digit
    uint64_t same = __ballot(has);
    for (uint32_t b = 0; b < p.bits; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t ones = __ballot(one);
      same &= one ? ones : ~ones;
    }
    const uint32_t rank = uint32_t(__popcll(same & ((uint64_t(1) << lane) - 1)));
    uint32_t to = 0;
    if (has) to = at[wave][d] + rank;
    wave_sync();
    if (has && rank == 0) at[wave][d] = to + uint32_t(__popcll(same));
    wave_sync();
    if (has) {
      keys[to] = key;
      order[to] = p.keys ? p.order[i] : i;
    }
  }
}

// ---------------------------------------------------------------------------
// Sums

constexpr uint32_t kSumThreads = 256;
constexpr uint32_t kSumWaves = kSumThreads / kWave;
constexpr uint32_t kBatch = 4;  // rows in flight per wavefront

struct SumArgs {
  const uint32_t *keys, *order;
  float* parts;      // [chunk][2][cols]: 0 of the run that came in, 1 of the run that goes on
  uint32_t n, rows, cols, accumulate;
  uint32_t chunk, chunks, slabs;
  uint32_t sum_wgs;  // workgroups that sum; the rest write the rows of no token
  float scale;
  Drop drop;
};

__device__ __forceinline__ void write_row(const SumArgs& a, const Mat<float>& out, uint32_t row, uint64_t col,
                                          uint32_t width, const float (&sum)[8]) {
  float* to = out.p + int64_t(row) * out.ld + col;
  Raw8<float> before;
  before.zero();
  if (a.accumulate) before.load(to, width);
  float v[8];
  before.widen(v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += sum[e] * a.scale;
  store8(to, width, v);
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

// Zeros in the rows of no token, a wavefront per row.
__device__ __forceinline__ void fill_rows(const SumArgs& a, const Mat<float>& out) {
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t waves = (gridDim.x - a.sum_wgs) * kSumWaves;
  for (uint32_t r = (blockIdx.x - a.sum_wgs) * kSumWaves + threadIdx.x / kWave; r < a.rows; r += waves) {
    const uint32_t at = lower_bound(a.keys, a.n, r, lane);
    if (at < a.n && a.keys[at] == r) continue;
    const float zero[8] = {};
    for (uint64_t col = lane * kBlockCols; col < a.cols; col += kWave * kBlockCols)
      store8(out.p + int64_t(r) * out.ld + col, uint32_t(a.cols - col < kBlockCols ? a.cols - col : kBlockCols), zero);
  }
}

template <typename T, bool kDrop>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(SumArgs a, Mat<const T> grad, Mat<float> out) {
  if (blockIdx.x >= a.sum_wgs) {
    fill_rows(a, out);
    return;
  }
  const uint32_t lane = threadIdx.x % kWave;
  const uint32_t job = __builtin_amdgcn_readfirstlane(blockIdx.x * kSumWaves + threadIdx.x / kWave);
  const uint32_t chunk = job / a.slabs;
  if (chunk >= a.chunks) return;
  const uint32_t block = (job - chunk * a.slabs) * kWave + lane;
  const uint64_t col = uint64_t(block) * kBlockCols;
  if (col >= a.cols) return;
  const uint32_t width = uint32_t(a.cols - col < kBlockCols ? a.cols - col : kBlockCols);
  const uint32_t lo = chunk * a.chunk, hi = min(a.n, lo + a.chunk);
  uint32_t run = a.keys[lo];
  bool came = lo > 0 && a.keys[lo - 1] == run;  // the run began in an earlier chunk
  float* parts = a.parts + uint64_t(chunk) * 2 * a.cols + col;
  float sum[8] = {};
  for (uint32_t at = lo; at < hi && run < a.rows; at += kBatch) {
    uint32_t key[kBatch], i[kBatch];
    Raw8<T> raw[kBatch];
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
      const uint32_t x = min(at + b, hi - 1);
      key[b] = at + b < hi ? a.keys[x] : kNone;
      i[b] = a.order[x];
      raw[b].load(grad.p + int64_t(i[b]) * grad.ld + col, width);
    }
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
      if (key[b] == kNone) break;
      if (key[b] != run) {
        if (came) store8(parts, width, sum);
        else write_row(a, out, run, col, width, sum);
        came = false;
        run = key[b];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
        if (run >= a.rows) break;  // from here on, ids outside the table
      }
      uint32_t bits[4];
      if (kDrop) a.drop.bits(i[b], block, bits);
      float v[8];
      raw[b].widen(v);
      if (kDrop) a.drop.apply(bits, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
  }
  if (run >= a.rows) return;
  if (came) store8(parts, width, sum);
  else if (hi < a.n && a.keys[hi] == run) store8(parts + a.cols, width, sum);
  else write_row(a, out, run, col, width, sum);
}

// Joins the parts of the run that begins in this chunk and goes on in the next
// ones: a workgroup per chunk and slab, its wavefronts taking the parts in turn.
__global__ __launch_bounds__(kSumThreads) void join_kernel(SumArgs a, Mat<float> out) {
  __shared__ float shared[kSumWaves][kWave][8];
  const uint32_t chunk = blockIdx.x / a.slabs, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t lo = chunk * a.chunk, hi = lo + a.chunk;  // not the last chunk
  const uint32_t run = a.keys[hi - 1];
  if (run >= a.rows || a.keys[hi] != run) return;
  if (a.keys[lo] == run && lo > 0 && a.keys[lo - 1] == run) return;  // it began before this chunk
  // the chunks that the run reaches: those whose first key is the run's
  uint32_t parts = 0;
  for (;;) {
    const uint32_t next = chunk + 1 + parts + lane;
    const bool on = next < a.chunks && a.keys[next * a.chunk] == run;
    const uint32_t more = uint32_t(__popcll(__ballot(on)));
    parts += more;
    if (more < kWave) break;
  }
  const uint64_t col = (uint64_t(blockIdx.x - chunk * a.slabs) * kWave + lane) * kBlockCols;
  const uint32_t width = col >= a.cols ? 0 : uint32_t(a.cols - col < kBlockCols ? a.cols - col : kBlockCols);
  float sum[8] = {};
  if (width) {
    // part 0 is this chunk's own
    for (uint32_t k = wave; k <= parts; k += kSumWaves) {
      Raw8<float> part;
      part.load(a.parts + (uint64_t(chunk + k) * 2 + (k == 0)) * a.cols + col, width);
      float v[8];
      part.widen(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) shared[wave][lane][e] = sum[e];
  __syncthreads();
  if (wave != 0 || !width) return;
#pragma unroll
  for (uint32_t w = 1; w < kSumWaves; ++w)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += shared[w][lane][e];
  write_row(a, out, run, col, width, sum);
}

// ---------------------------------------------------------------------------

constexpr uint32_t kRankMost = 8192;  // tokens that are ordered by counting

uint32_t slabs_of(uint64_t cols) { return uint32_t((cols + kWave * kBlockCols - 1) / (kWave * kBlockCols)); }

// Tokens per chunk: at most kJobs wavefronts in all, but 4 to 128 tokens each.
constexpr uint64_t kJobs = 4096, kChunkLeast = 4, kChunkMost = 128;

uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

uint32_t chunk_of(uint64_t n, uint64_t cols) {
  return uint32_t(std::min(kChunkMost, std::max(kChunkLeast, up(n * slabs_of(cols), kJobs))));
}

// Columns of parts, at most, over all chunks: n / kChunkLeast of them, or where
// chunks are longer kJobs / slabs, or where those would pass kChunkMost tokens
// n / kChunkMost.  It grows with n and cols, so a workspace serves smaller calls.
uint64_t part_cols(uint64_t n, uint64_t cols) {
  return std::min(up(n, kChunkLeast) * cols, std::max(kJobs * kWave * kBlockCols + cols, up(n, kChunkMost) * cols));
}

hipError_t sort_tokens(const Tokens& t, char* work, const EmbedGradSizes& w, const uint32_t** keys,
                       const uint32_t** order, hipStream_t stream) {
  auto at = [&](uint64_t byte) { return reinterpret_cast<uint32_t*>(work + byte); };
  *keys = at(w.keys[0]);
  *order = at(w.order[0]);
  if (t.n <= kRankMost) {
    hipLaunchKernelGGL(rank_kernel, dim3((t.n + kWave - 1) / kWave), dim3(kRankWaves * kWave), 0, stream, t,
                       at(w.keys[0]), at(w.order[0]));
    return hipGetLastError();
  }
  uint32_t bits = 1;
  while (bits < 32 && t.rows >> bits) ++bits;  // of the largest key, `rows`
  const uint32_t passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
  SortPass p{};
  p.tile = (t.n + kMaxTiles - 1) / kMaxTiles;
  p.tile = std::max(1024u, (p.tile + kSortThreads - 1) / kSortThreads * kSortThreads);
  p.tiles = (t.n + p.tile - 1) / p.tile;
  for (uint32_t k = 0; k < passes; ++k) {
    p.shift = bits * k / passes;
    p.bits = bits * (k + 1) / passes - p.shift;
    uint32_t *to_keys = at(w.keys[k % 2]), *to_order = at(w.order[k % 2]);
    hipLaunchKernelGGL(digit_kernel, dim3(p.tiles), dim3(kSortThreads), 0, stream, t, p, at(w.counts));
    hipLaunchKernelGGL(move_kernel, dim3(p.tiles), dim3(kSortThreads), 0, stream, t, p, at(w.counts), to_keys, to_order);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    *keys = p.keys = to_keys;
    *order = p.order = to_order;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch(const etc_embed_grad_args& x, const Drop& drop, hipStream_t stream) {
  const uint32_t n = uint32_t(x.tokens.count), rows = uint32_t(x.dtable.rows), cols = uint32_t(x.dtable.cols);
  const EmbedGradSizes w = embed_grad_sizes(n, rows, cols);
  char* work = static_cast<char*>(x.workspace);
  SumArgs a{};
  if (n) {
    const Tokens t{Ids{x.tokens.data, x.tokens.dtype == ETC_IDS_I64}, x.row0, rows, n};
    const hipError_t e = sort_tokens(t, work, w, &a.keys, &a.order, stream);
    if (e != hipSuccess) return e;
  }
  a.parts = reinterpret_cast<float*>(work + w.parts);
  a.n = n;
  a.rows = rows;
  a.cols = cols;
  a.accumulate = x.accumulate != 0;
  a.chunk = chunk_of(n, cols);
  a.chunks = (n + a.chunk - 1) / a.chunk;
  a.slabs = slabs_of(cols);
  a.sum_wgs = uint32_t((uint64_t(a.chunks) * a.slabs + kSumWaves - 1) / kSumWaves);
  a.scale = float(x.scale);
  a.drop = drop;
  const Mat<const T> grad{static_cast<const T*>(x.grad.data), x.grad.ld};
  const Mat<float> out{static_cast<float*>(x.dtable.data), x.dtable.ld};
  const uint32_t fill_wgs = a.accumulate ? 0 : std::min((rows + kSumWaves - 1) / kSumWaves, 1u << 20);
  const dim3 wgs(a.sum_wgs + fill_wgs), block(kSumThreads);
  if (drop.limit) hipLaunchKernelGGL((sum_kernel<T, true>), wgs, block, 0, stream, a, grad, out);
  else hipLaunchKernelGGL((sum_kernel<T, false>), wgs, block, 0, stream, a, grad, out);
  if (a.chunks > 1) hipLaunchKernelGGL(join_kernel, dim3((a.chunks - 1) * a.slabs), block, 0, stream, a, out);
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
  w.keys[0] = take(4 * n);
  w.order[0] = take(4 * n);
  if (n > kRankMost) {
    w.keys[1] = take(4 * n);
    w.order[1] = take(4 * n);
    w.counts = take((uint64_t(4) << kMaxDigitBits) * kMaxTiles);
  }
  w.parts = take(part_cols(n, cols) * 2 * sizeof(float));
  return w;
}

bool embed_grad_fits(uint64_t n, uint64_t cols) {
  // a workgroup per chunk and slab in the largest launch, of kSumThreads each
  return up(n, chunk_of(n, cols)) * slabs_of(cols) <= (uint64_t(1) << 32) / kSumThreads / 2;
}

hipError_t launch_embed_grad(const etc_embed_grad_args& a, const Drop& drop, hipStream_t stream) {
  return a.grad.dtype == ETC_DTYPE_F32 ? launch<float>(a, drop, stream) : launch<bf16>(a, drop, stream);
}

}  // namespace etc
