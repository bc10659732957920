// matmul8.hip -- products of 8-bit integers with a scale for each row of either
// operand (etc_matmul8).
//
//   out[m, n] = sx[m] sw[n] (sum over k of x[m, k] w[n, k]) + bias[n]
//
// The sums are exact in 32-bit integers, so how they are split changes no bit.
//
// Three kernels: few rows (1 x 12288 x 4096: 10.3 us, 4.9 TB/s of weights, where a kernel that only reads
// them takes 8.9), tiles whose sums are split over wavefronts (512 x 4096 x 4096: 18.6 us) and tiles of
// quarters (8192 x 22016 x 4096: 664 to 750 us with the card, 2.0 to 2.2 POP/s).  The first waits for HBM, the middle one for
// what its CUs read into their LDS.  The last has two bounds.  Power holds the clock at 1.6 to 1.9 GHz: operands of zeros take as
// many cycles at 2.3 (4096 x 4096 x 16384: 178 us, 230 with random ones).  And its matrix pipes are busy for 54 % of the cycles (64 %
// there): in 7 % of them a CU has no wavefront (9 %), wavefronts wait for loads, LDS and barriers in 13 % of their time (10 %), and
// a wavefront to a SIMD leaves nobody to fill the pipe while it issues what stands between matrix instructions.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "eight.hpp"

namespace etc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct Product {
  const uint8_t *x, *w;
  int64_t xld, wld;
  const float *sx, *sw;
  int64_t sxld, swld;  // from a row's scale to the next one's
  uint32_t m, n, k;
  void* out;
  int64_t ld;
  const void* bias;

  __device__ __forceinline__ float x_scale(uint32_t i) const { return sx ? sx[int64_t(i) * sxld] : 1.0f; }
  __device__ __forceinline__ float w_scale(uint32_t j) const { return sw ? sw[int64_t(j) * swld] : 1.0f; }
  template <typename T>
  __device__ __forceinline__ float bias_of(uint64_t j) const {
    return bias ? float(static_cast<const T*>(bias)[j]) : -0.0f;  // which leaves every number as it is
  }
};

// An element of the output from its sum, the same in all kernels to the bit.
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale, float bias) {
  return __builtin_fmaf(float(sum) * x_scale, w_scale, bias);
}

// Four neighbouring columns n .. n + 3 of row m, as far as there are any.
template <typename T>
__device__ __forceinline__ void store4(const Product& p, uint32_t m, uint64_t n, const int* sums, float x_scale) {
  const uint32_t width = n >= p.n ? 0 : uint32_t(min(uint64_t(4), p.n - n));
  float v[4];
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e) {
    if (e >= width) break;
    v[e] = scaled(sums[e], x_scale, p.w_scale(uint32_t(n) + e), p.bias_of<T>(n + e));
  }
  T* out = static_cast<T*>(p.out) + int64_t(m) * p.ld + int64_t(n);
  Raw<T, 4, false> raw;
  raw.narrow(v);
  if (width) raw.store(out, width);
}

// Operands stand in LDS as rows of 128 columns, whose 8 chunks of 16 bytes are
// permuted: row r has chunk c at place c ^ (r / 2 % 8), so that reads of one chunk of 16
// rows touch all 64 banks once.  They come straight from memory (`direct`, 16 bytes a lane
// at multiples of 16, 8 rows to an instruction, whose lanes take the chunks in the order
// of their places), or by way of registers.  Neighbouring lanes have neighbouring
// chunks: fragments of matrix instructions, whose neighbours are rows, took four times as long to load.
constexpr uint32_t kDepth = 128;
constexpr uint32_t kCus = 256;

// The column in its row of the chunk that lane `lane` of the load of rows 8 g .. 8 g + 7 fills; the other
// parity of g has it flipped by 64.
__device__ __forceinline__ uint32_t chunk_of(uint32_t lane, uint32_t g) { return (lane % 8 ^ (lane / 16 + g % 2 * 4)) * 16; }

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

__device__ __forceinline__ void load_direct(const uint8_t* from, uint8_t* to) {
  __builtin_amdgcn_global_load_lds((global_void*)from, (lds_void*)to, 16, 0, 0);
}

__device__ __forceinline__ void place16(uint8_t* to, const Raw8<16, false>& r) {
  *reinterpret_cast<i32x4*>(to) = i32x4{int(r.w[0]), int(r.w[1]), int(r.w[2]), int(r.w[3])};
}

// The 16 bytes from column k of the row at p on, zeros past `end`.
__device__ __forceinline__ void load_tail(Raw8<16, false>& r, const uint8_t* p, uint64_t k, uint32_t end) {
  const uint32_t width = block_width<16>(k, end);
  r.zero();
  if (width) r.load(p + k, width, end < 16);
  r.shift(width);
}

// ---------------------------------------------------------------------------
// Few rows: everything waits for the weights.  A workgroup has 16 columns of the
// output and kG groups of 8 rows; its wavefronts share the sums' length between
// them, each with kAhead stages of 128 columns on their way into LDS of its own, and add
// up at the end.  Slots of a wavefront's own need no barrier; kAhead stages of at most 16 wavefronts fill
// the LDS, which is what keeps HBM's queues full.

template <uint32_t kG>
constexpr uint32_t kAhead = kG == 1 ? 4 : kG == 2 ? 3 : 2;
template <uint32_t kG>
constexpr uint32_t kStage = (2 + kG) * 1024;  // bytes: 16 rows of w, 8 kG of x
template <uint32_t kG>
constexpr uint32_t kFewWaves = kG == 1 ? 6 : kG < 6 ? 16 : 8;  // at most

template <uint32_t kG, bool kDirect>
__global__ __launch_bounds__(kFewWaves<kG> * 64) void matmul8_few_kernel(Product p, uint32_t wide, uint32_t across) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t memory[];
  constexpr uint32_t kM = (kG + 1) / 2, kLoads = 2 + kG, kSlots = kAhead<kG>;
  const uint32_t lane = threadIdx.x % 64, waves = blockDim.x / 64;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t down = blockIdx.x / across, m0 = down * kG * 8;
  const uint64_t n0 = uint64_t(blockIdx.x - down * across) * 16;
  if (n0 >= p.n) return;
  uint8_t* slots = memory + wave * kSlots * kStage<kG>;
  // rows past the end repeat the last one; what comes of them is not stored
  const uint32_t chunks[2] = {chunk_of(lane, 0), chunk_of(lane, 1)};  // of w's and x's loads alike: both begin with an even one
  const uint8_t* rows[kLoads];
#pragma unroll
  for (uint32_t i = 0; i < kLoads; ++i)
    rows[i] = i < 2 ? p.w + int64_t(min(n0 + i * 8 + lane / 8, uint64_t(p.n) - 1)) * p.wld
                    : p.x + int64_t(min(m0 + (i - 2) * 8 + lane / 8, p.m - 1)) * p.xld;
  const uint32_t whole = p.k / kDepth;
  // the columns past whole stages are the last wavefront's, loaded first and multiplied last
  const bool rest = wave == waves - 1 && p.k % kDepth;
  Raw8<16, false> tail[kLoads];
  auto tail_width = [&](uint32_t i) { return block_width<16>(uint64_t(whole) * kDepth + chunks[i % 2], p.k); };
  if (rest) {
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      tail[i].zero();
      if (tail_width(i)) tail[i].load(rows[i] + uint64_t(whole) * kDepth + chunks[i % 2], tail_width(i), p.k < 16);
    }
    compiler_fence();
  }
  const uint32_t from = uint32_t(uint64_t(whole) * wave / waves), to = uint32_t(uint64_t(whole) * (wave + 1) / waves);

  i32x4 acc[kM] = {};
  const uint32_t at = lane % 16 * kDepth + (lane / 16 ^ lane / 2 % 8) * 16;
  auto multiply = [&](const uint8_t* slot) {
#pragma unroll
    for (uint32_t step = 0; step < 2; ++step) {
      const i32x4 w = *reinterpret_cast<const i32x4*>(slot + (at ^ step * 64));
#pragma unroll
      for (uint32_t t = 0; t < kM; ++t) {
        // of a last group of 8 rows, lanes 8 .. 15 read the same again
        const uint32_t row = kG % 2 && t == kM - 1 ? (at & ~(8 * kDepth)) ^ (at & 8 * kDepth) / (8 * kDepth) * 64 : at;
        const i32x4 x = *reinterpret_cast<const i32x4*>(slot + 2048 + t * 2048 + (row ^ step * 64));
        acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc[t], 0, 0, 0);
      }
    }
  };
  if constexpr (kDirect) {
    auto start = [&](uint32_t s) {
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i) load_direct(rows[i] + uint64_t(s) * kDepth + chunks[i % 2], slots + s % kSlots * kStage<kG> + i * 1024);
    };
    const uint32_t first = min(from + kSlots, to);
    for (uint32_t s = from; s < first; ++s) start(s);
    for (uint32_t s = from; s < to; ++s) {
      // the oldest stage has arrived where at most the loads of kSlots - 1 later ones are under way
      if (s + kSlots <= to) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads * (kSlots - 1)) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      multiply(slots + s % kSlots * kStage<kG>);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
      if (s + kSlots < to) start(s + kSlots);
    }
  } else {
    for (uint32_t s0 = from; s0 < to; s0 += kSlots) {
      Raw8<16, false> r[kSlots][kLoads];
#pragma unroll
      for (uint32_t b = 0; b < kSlots; ++b) {
        if (s0 + b >= to) break;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) r[b][i].load(rows[i] + uint64_t(s0 + b) * kDepth + chunks[i % 2], 16, false);
      }
      compiler_fence();
#pragma unroll
      for (uint32_t b = 0; b < kSlots; ++b) {
        if (s0 + b >= to) break;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) place16(slots + b * kStage<kG> + i * 1024 + lane * 16, r[b][i]);
        multiply(slots + b * kStage<kG>);
      }
    }
  }
  if (rest) {
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      tail[i].shift(tail_width(i));
      place16(slots + i * 1024 + lane * 16, tail[i]);
    }
    multiply(slots);
  }
  __syncthreads();
  i32x4* parts = reinterpret_cast<i32x4*>(memory);  // [wavefront][kM][lane]
#pragma unroll
  for (uint32_t t = 0; t < kM; ++t) parts[(wave * kM + t) * 64 + lane] = acc[t];
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < kM * 64; e += blockDim.x) {
    i32x4 sum = parts[e];
    for (uint32_t v = 1; v < waves; ++v) sum += parts[v * kM * 64 + e];
    const uint32_t m = m0 + e / 64 * 16 + e % 16;
    if (e / 64 * 16 + e % 16 >= kG * 8 || m >= p.m) continue;
    const int sums[4] = {sum[0], sum[1], sum[2], sum[3]};
    const uint64_t n = n0 + e % 64 / 16 * 4;
    if (wide) store4<float>(p, m, n, sums, p.x_scale(m));
    else store4<bf16>(p, m, n, sums, p.x_scale(m));
  }
}

// ---------------------------------------------------------------------------
// Tiles of 64 kF x 64 kF of the output by four wavefronts, each of which has a
// quarter in registers.  Stages of 128 columns of the operands stand in kCopies parts of the LDS:
// while one is multiplied the others are filled, straight from memory
// (kDirect: rows at multiples of 16 bytes), or two parts in turn by way of registers, which
// hold the kSets stages behind.
// In a stage the loads of a later one, the matrix instructions and the reads of the next step's operands
// stand in the order written here: a wavefront that has its CU's registers to itself has nobody to hide its
// waits.  256 x 256 reads 1 byte for 128 multiplications, 128 x 128 for 64; stages of 64 columns, of which
// four or five fit, took 4 % more (half lines of memory, twice the barriers).

template <uint32_t... kS, typename F>
__device__ __forceinline__ void for_each_below(std::integer_sequence<uint32_t, kS...>, F f) {
  (f(std::integral_constant<uint32_t, kS>()), ...);
}

struct Tiles {
  uint32_t m, n;  // tiles down and across
  uint32_t count;
};

// Workgroups are dealt to the 8 XCDs in turn.  An XCD has a run of tiles, ordered
// in bands of 8 tiles down, so that those that it works on at once share rows in its L2.
__device__ __forceinline__ void place_tile(const Tiles& t, uint32_t* tm, uint32_t* tn) {
  constexpr uint32_t kXcds = 8, kBand = 8;
  const uint32_t xcd = blockIdx.x % kXcds, each = t.count / kXcds, more = t.count % kXcds;
  const uint32_t at = xcd * each + min(xcd, more) + blockIdx.x / kXcds;
  const uint32_t band = at / (kBand * t.n), rest = at - band * kBand * t.n;
  const uint32_t down = min(kBand, t.m - band * kBand);
  *tn = rest / down;
  *tm = band * kBand + rest - *tn * down;
}

template <typename T, uint32_t kF, uint32_t kCopies, bool kDirect>
__global__ __launch_bounds__(256, kF == 4 || kCopies == 4 ? 1 : 2) void matmul8_tile_kernel(Product p, Tiles tiles) {
  constexpr uint32_t kTile = 64 * kF;
  constexpr uint32_t kLoads = kTile / 32;  // of a wavefront, of 8 rows each, for one operand; even, so that load i's parity is its rows'
  constexpr uint32_t kOperand = kTile * kDepth, kCopy = 2 * kOperand;
  __shared__ __attribute__((aligned(1024))) uint8_t buffer[kCopies * kCopy];  // of x's and w's rows
  uint32_t tm, tn;
  place_tile(tiles, &tm, &tn);
  const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint64_t m0 = uint64_t(tm) * kTile, n0 = uint64_t(tn) * kTile;
  const uint8_t* base[2] = {p.x + int64_t(m0) * p.xld, p.w + int64_t(n0) * p.wld};
  uint32_t offset[2][kLoads];
  const uint32_t chunks[2] = {chunk_of(lane, 0), chunk_of(lane, 1)};
#pragma unroll
  for (uint32_t i = 0; i < kLoads; ++i) {  // rows past the end repeat the last one
    const uint64_t row = (wave * kLoads + i) * 8 + lane / 8;
    offset[0][i] = uint32_t(min(row, p.m - 1 - m0)) * uint32_t(p.xld) + chunks[i % 2];
    offset[1][i] = uint32_t(min(row, p.n - 1 - n0)) * uint32_t(p.wld) + chunks[i % 2];
  }
  // (kF = 2 by way of registers spills 27 of its 256, 112 bytes a lane)
  constexpr uint32_t kSets = kDirect || kF == 4 ? 1 : 2;
  constexpr uint32_t kFar = kDirect ? kCopies - 1 : kSets;  // stages between one that starts and the one that is multiplied
  Raw8<16, false> staged[kSets][2][kLoads];
  // load `i` of operand o, of 128 columns from k on, into copy c or on its way there in registers
  auto start = [&](uint64_t k, uint32_t c, auto set, uint32_t o, uint32_t i) {
    if constexpr (kDirect)
      load_direct(base[o] + k + offset[o][i], &buffer[c * kCopy + o * kOperand + (wave * kLoads + i) * 1024]);
    else staged[set()][o][i].load(base[o] + k + offset[o][i], 16, false);
  };
  auto place = [&](uint32_t c, auto set) {
#pragma unroll
    for (uint32_t o = 0; o < 2; ++o) {
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i)
        place16(&buffer[c * kCopy + o * kOperand + (wave * kLoads + i) * 1024 + lane * 16], staged[set()][o][i]);
    }
  };
  using Zero = std::integral_constant<uint32_t, 0>;
  // until all wavefronts have filled their part of a copy, with at most `later` direct loads of others under way
  auto finish = [&](uint32_t c, auto set, auto later) {
    if constexpr (kDirect) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(later)::value) : "memory");
    } else {
      place(c, set);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
  };

  const uint32_t left[2] = {wave % 2 * (kTile / 2), wave / 2 * (kTile / 2)};  // the wavefront's rows of x and of w
  uint32_t place0[2];  // of a lane's operand in the first step; in step s, s * 32 is added to its chunk's place
#pragma unroll
  for (uint32_t o = 0; o < 2; ++o) place0[o] = o * kOperand + (left[o] + lane % 32) * kDepth + (lane / 32 ^ lane / 2 % 8) * 16;
  auto read = [&](uint32_t c, uint32_t step, uint32_t o, uint32_t b) {
    return *reinterpret_cast<const i32x4*>(&buffer[c * kCopy + (place0[o] ^ step * 32) + b * 32 * kDepth]);
  };

  i32x16 acc[kF][kF] = {};  // [of w][of x]
  i32x4 x[2][kF], w[2][kF];
  // Multiplies copy c, whose first operands are in x[0] and w[0].  kMore: leaves those of the next copy there.
  // kFill: meanwhile starts the stage from column k on, into the copy before (kDirect) or into register set
  // kSet, whose stage has been placed; the next stage is in the set behind it.  The order is kept as it
  // stands: loads, and reads of the next step's operands, one by one between matrix instructions.
  auto multiply = [&](uint32_t c, auto set, auto fill, auto more, uint64_t k) {
    constexpr bool kFill = decltype(fill)::value, kMore = decltype(more)::value;
    constexpr uint32_t kEach = kF * kF, kReads = 2 * kF, kSet = decltype(set)::value;
    using Behind = std::integral_constant<uint32_t, (kSet + 1) % kSets>;
    const uint32_t after = c + 1 == kCopies ? 0 : c + 1, before = c ? c - 1 : kCopies - 1;
#pragma unroll
    for (uint32_t step = 0; step < 4; ++step) {
      const uint32_t now = step % 2, next = 1 - now;
#pragma unroll
      for (uint32_t q = 0; q < kEach; ++q) {
        if (kFill && step == 0) {
#pragma unroll
          for (uint32_t d = q * 2 * kLoads / kEach; d < (q + 1) * 2 * kLoads / kEach; ++d) start(k, before, set, d / kLoads, d % kLoads);
        }
        if (kMore && step == 3 && q == kEach / 2)
          finish(after, Behind(), std::integral_constant<uint32_t, kFill ? (kCopies - 2) * 2 * kLoads : 0>());
        __builtin_amdgcn_sched_barrier(0);
        acc[q / kF][q % kF] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[now][q / kF], x[now][q % kF], acc[q / kF][q % kF], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t r = 0; r < kReads; ++r) {
          const uint32_t b = r / 2, o = 1 - r % 2;
          i32x4& to = o ? w[next][b] : x[next][b];
          if (step < 3 && r * kEach * 3 / (4 * kReads) == q) to = read(c, step + 1, o, b);
          if (kMore && step == 3 && kEach / 2 + r * (kEach - kEach / 2) * 3 / (4 * kReads) == q) to = read(after, 0, o, b);
        }
      }
    }
  };

  // The columns past whole stages come first, so that the loop has whole ones only.
  const uint32_t rest = p.k % kDepth != 0, stages = p.k / kDepth + rest;
  if (stages) {
    if (rest) {
#pragma unroll
      for (uint32_t o = 0; o < 2; ++o) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i)
          load_tail(staged[0][o][i], base[o] + offset[o][i] - chunks[i % 2], uint64_t(stages - 1) * kDepth + chunks[i % 2], p.k);
      }
      if (kDirect) place(0, Zero());
    }
    auto column = [&](uint32_t s) { return uint64_t(s - rest) * kDepth; };
    // stage s's copy, and its register set
    auto start_stage = [&](auto s) {
      constexpr uint32_t kS = decltype(s)::value;
      if (kS < rest || kS >= stages) return;
#pragma unroll
      for (uint32_t o = 0; o < 2; ++o) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) start(column(kS), kS % kCopies, std::integral_constant<uint32_t, kS % kSets>(), o, i);
      }
    };
    for_each_below(std::make_integer_sequence<uint32_t, kFar>(), start_stage);
    finish(0, Zero(), Zero());
#pragma unroll
    for (uint32_t b = 0; b < kF; ++b) x[0][b] = read(0, 0, 0, b), w[0][b] = read(0, 0, 1, b);
    uint32_t s = 0, c = 0;
    auto next_copy = [&] { c = c + 1 == kCopies ? 0 : c + 1; };
    if constexpr (kSets == 1) {
      for (; s + kFar < stages; ++s, next_copy()) multiply(c, Zero(), std::true_type(), std::true_type(), column(s + kFar));
      for (; s + 1 < stages; ++s, next_copy()) multiply(c, Zero(), std::false_type(), std::true_type(), 0);
      multiply(c, Zero(), std::false_type(), std::false_type(), 0);
    } else {  // in rounds of kSets stages, whose registers are named in the code
      auto turn = [&](auto set, auto sure) {
        if (decltype(sure)::value || s + kFar < stages) multiply(c, set, std::true_type(), std::true_type(), column(s + kFar));
        else if (s + 1 < stages) multiply(c, set, std::false_type(), std::true_type(), 0);
        else if (s < stages) multiply(c, set, std::false_type(), std::false_type(), 0);
        ++s;
        next_copy();
      };
      auto round = [&](auto sure) {
        turn(Zero(), sure);
        turn(std::integral_constant<uint32_t, 1>(), sure);
      };
      while (s + kFar + kSets <= stages) round(std::true_type());
      while (s < stages) round(std::false_type());
    }
  }
  // Each wavefront turns 32 rows of its quarter at a time round in a part of the
  // LDS of its own, so that it stores whole rows of 32 kF columns.
  constexpr uint32_t kC = kLaneCols<T>, kCols = 32 * kF, kPitch = kCols * sizeof(T) + 16;
  static_assert(4 * 32 * kPitch <= sizeof buffer, "LDS");
  uint8_t* part = buffer + wave * 32 * kPitch;
  float scale_w[kF][16], bias[kF][16];
  const uint64_t n1 = n0 + left[1], m1 = m0 + left[0];
#pragma unroll
  for (uint32_t i = 0; i < kF; ++i) {
#pragma unroll
    for (uint32_t e = 0; e < 16; ++e) {
      const uint64_t n = min(n1 + i * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4, uint64_t(p.n) - 1);
      scale_w[i][e] = p.w_scale(uint32_t(n));
      bias[i][e] = p.bias_of<T>(n);
    }
  }
  __syncthreads();  // all have read their operands
#pragma unroll
  for (uint32_t j = 0; j < kF; ++j) {
    const float scale_x = p.x_scale(uint32_t(min(m1 + j * 32 + lane % 32, uint64_t(p.m) - 1)));
#pragma unroll
    for (uint32_t i = 0; i < kF; ++i) {
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
          v[e] = scaled(acc[i][j][4 * q + e], scale_x, scale_w[i][4 * q + e], bias[i][4 * q + e]);
        store_block<true>(reinterpret_cast<T*>(part + lane % 32 * kPitch) + i * 32 + q * 8 + lane / 32 * 4, 4, v);
      }
    }
    constexpr uint32_t kAcross = kCols / kC, kDown = 64 / kAcross;  // lanes to a row, rows at a time
#pragma unroll
    for (uint32_t u = 0; u < 32 / kDown; ++u) {
      const uint32_t r = u * kDown + lane / kAcross;
      const uint64_t m = m1 + j * 32 + r, n = n1 + lane % kAcross * kC;
      Raw<T, kC, false> raw;
      raw.load(reinterpret_cast<const T*>(part + r * kPitch) + lane % kAcross * kC, kC, false);
      if (m < p.m && n < p.n) raw.template store<true>(static_cast<T*>(p.out) + int64_t(m) * p.ld + int64_t(n), block_width<kC>(n, p.n));
    }
  }
}

// ---------------------------------------------------------------------------
// Tiles of 32 kA x 32 kB where larger ones would leave CUs idle.  Each of the four
// wavefronts has the whole tile, for one of the four steps of 32 columns in each
// stage: kA kB matrix instructions to kA + kB reads, where a quarter of a tile of 64 x 64 each had one to two
// and waited for LDS.  The wavefronts' sums are added up in LDS at the end.
// 128 x 4096 x 4096: 9.1 us, 200 rows 11.1, 512 18.6, 1024 23.5 (1.5 POP/s).  Rows that lie
// at no multiples of 16 bytes go by way of registers: loads at odd addresses run at a third of the rate (200 x 4096 x 4095: 19.9).

template <typename T, uint32_t kA, uint32_t kB, bool kDirect>
__global__ __launch_bounds__(256, kDirect && kA * kB <= 4 ? 2 : 1) void matmul8_split_kernel(Product p, Tiles tiles) {
  constexpr uint32_t kStageBytes = (kA + kB) * 32 * kDepth, kLoads = kA + kB;  // loads of a wavefront, of 8 rows each
  // stages in LDS; behind them, in registers (kDirect: none)
  constexpr uint32_t kCopies = kDirect ? 4 : 2, kSets = kA * kB > 4 ? 2 : 3;
  constexpr uint32_t kRows = 32 * kA, kCols = 32 * kB, kPitch = kCols * 4 + 16;
  __shared__ __attribute__((aligned(1024))) uint8_t buffer[std::max(4 * kRows * kPitch, kCopies * kStageBytes)];
  uint32_t tm, tn;
  place_tile(tiles, &tm, &tn);
  const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint64_t m0 = uint64_t(tm) * kRows, n0 = uint64_t(tn) * kCols;
  const uint8_t* rows[kLoads];  // kA of x, then kB of w
#pragma unroll
  for (uint32_t i = 0; i < kLoads; ++i) {
    const uint32_t row = (wave * (i < kA ? kA : kB) + (i < kA ? i : i - kA)) * 8 + lane / 8;  // rows past the end repeat the last one
    rows[i] = i < kA ? p.x + int64_t(min(m0 + row, uint64_t(p.m) - 1)) * p.xld : p.w + int64_t(min(n0 + row, uint64_t(p.n) - 1)) * p.wld;
  }
  // of loads of an even group of 8 rows and of an odd one
  const uint32_t chunks[2] = {chunk_of(lane, 0), chunk_of(lane, 1)};
  auto chunk = [&](uint32_t i) { return chunks[(i < kA ? wave * kA + i : wave * kB + i - kA) % 2]; };
  const uint32_t rest = p.k % kDepth != 0, stages = p.k / kDepth + rest;
  auto target = [&](uint32_t s, uint32_t i) {
    return &buffer[s % kCopies * kStageBytes + (i < kA ? wave * kA + i : 4 * kA + wave * kB + i - kA) * 1024];
  };
  Raw8<16, false> staged[kSets][kLoads];
  auto start = [&](uint32_t s, auto set) {  // a stage of whole columns: those past whole stages come first
    const uint64_t k = uint64_t(s - rest) * kDepth;
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      if constexpr (kDirect) load_direct(rows[i] + k + chunk(i), target(s, i));
      else staged[set()][i].load(rows[i] + k + chunk(i), 16, false);
    }
  };
  auto place = [&](uint32_t s, auto set) {
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) place16(target(s, i) + lane * 16, staged[set()][i]);
  };
  const uint32_t at = lane % 32 * kDepth + ((wave * 2 + lane / 32) ^ lane / 2 % 8) * 16;
  i32x16 acc[kB][kA] = {};  // [of w][of x]
  i32x4 x[kA], w[kB];
  auto read = [&](uint32_t s) {
    const uint8_t* from = &buffer[s % kCopies * kStageBytes + at];
#pragma unroll
    for (uint32_t b = 0; b < kA; ++b) x[b] = *reinterpret_cast<const i32x4*>(from + b * 32 * kDepth);
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) w[b] = *reinterpret_cast<const i32x4*>(from + (kA + b) * 32 * kDepth);
  };
  using Zero = std::integral_constant<uint32_t, 0>;
  // Multiplies stage s, whose operands are in x and w, and reads stage s + 1 (which register set `next` holds) behind it.
  // kFill: starts a stage, into the copy that has been read or into the set that has been placed.
  auto turn = [&](uint32_t s, auto next, auto fill) {
    i32x4 u[kA], v[kB];
#pragma unroll
    for (uint32_t b = 0; b < kA; ++b) u[b] = x[b];
#pragma unroll
    for (uint32_t b = 0; b < kB; ++b) v[b] = w[b];
    constexpr bool kFill = decltype(fill)::value;
    if constexpr (kDirect) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kFill ? (kCopies - 2) * kLoads : 0) : "memory");
    } else {
      place(s + 1, next);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    read(s + 1);
    if constexpr (kFill) start(kDirect ? s + kCopies : s + 1 + kSets, next);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (uint32_t i = 0; i < kB; ++i) {
#pragma unroll
      for (uint32_t j = 0; j < kA; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(v[i], u[j], acc[i][j], 0, 0, 0);
    }
  };
  if (stages) {
    if (rest) {
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i) load_tail(staged[0][i], rows[i], uint64_t(stages - 1) * kDepth + chunk(i), p.k);
      if (kDirect) place(0, Zero());
    }
    for_each_below(std::make_integer_sequence<uint32_t, kDirect ? kCopies : kSets>(), [&](auto s) {
      if (s() >= rest && s() < stages) start(s(), std::integral_constant<uint32_t, s() % kSets>());
    });
    if constexpr (kDirect) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    } else {
      place(0, Zero());
      if (kSets < stages) start(kSets, Zero());
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    read(0);
    uint32_t s = 0;
    if constexpr (kDirect) {
      for (; s + kCopies < stages; ++s) turn(s, Zero(), std::true_type());
      for (; s + 1 < stages; ++s) turn(s, Zero(), std::false_type());
    } else {
      // in rounds of kSets stages, whose registers are named in the code: turn s places set (s + 1) % kSets
      for (; s + 2 * kSets < stages; s += kSets)
        for_each_below(std::make_integer_sequence<uint32_t, kSets>(),
                       [&](auto d) { turn(s + d(), std::integral_constant<uint32_t, (d() + 1) % kSets>(), std::true_type()); });
      for (; s + 1 < stages; s += kSets)
        for_each_below(std::make_integer_sequence<uint32_t, kSets>(), [&](auto d) {
          using Next = std::integral_constant<uint32_t, (d() + 1) % kSets>;
          if (s + d() + 1 + kSets < stages) turn(s + d(), Next(), std::true_type());
          else if (s + d() + 1 < stages) turn(s + d(), Next(), std::false_type());
        });
    }
#pragma unroll
    for (uint32_t i = 0; i < kB; ++i) {
#pragma unroll
      for (uint32_t j = 0; j < kA; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[i], x[j], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();  // all have read their operands
#pragma unroll
  for (uint32_t i = 0; i < kB; ++i) {
#pragma unroll
    for (uint32_t j = 0; j < kA; ++j) {
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q)
        *reinterpret_cast<i32x4*>(buffer + (wave * kRows + j * 32 + lane % 32) * kPitch + (i * 32 + q * 8 + lane / 32 * 4) * 4) =
            i32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    }
  }
  __syncthreads();
  constexpr uint32_t kC = kLaneCols<T>, kAcross = kCols / kC;  // lanes to a row
  for (uint32_t e = threadIdx.x; e < kRows * kAcross; e += 256) {
    const uint32_t r = e / kAcross, c = e % kAcross * kC;
    const uint64_t m = m0 + r, n = n0 + c;
    if (m >= p.m || n >= p.n) continue;
    const float scale_x = p.x_scale(uint32_t(m));
    float v[kC];
#pragma unroll
    for (uint32_t b = 0; b < kC; b += 4) {
      i32x4 sum = {};
#pragma unroll
      for (uint32_t f = 0; f < 4; ++f) sum += *reinterpret_cast<const i32x4*>(buffer + (f * kRows + r) * kPitch + (c + b) * 4);
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t column = uint32_t(min(n + b + k, uint64_t(p.n) - 1));
        v[b + k] = scaled(sum[k], scale_x, p.w_scale(column), p.bias_of<T>(column));
      }
    }
    store_block<false, true>(static_cast<T*>(p.out) + int64_t(m) * p.ld + int64_t(n), block_width<kC>(n, p.n), v);
  }
}

template <typename T, uint32_t kF, uint32_t kCopies, bool kDirect>
hipError_t launch_tiles(const Product& p, hipStream_t stream) {
  constexpr uint32_t kTile = 64 * kF;
  Tiles t{(p.m + kTile - 1) / kTile, (p.n + kTile - 1) / kTile, 0};
  t.count = t.m * t.n;
  hipLaunchKernelGGL((matmul8_tile_kernel<T, kF, kCopies, kDirect>), dim3(t.count), dim3(256), 0, stream, p, t);
  return hipGetLastError();
}

template <typename T, uint32_t kA, uint32_t kB>
hipError_t launch_split(const Product& p, bool direct, hipStream_t stream) {
  Tiles t{(p.m + 32 * kA - 1) / (32 * kA), (p.n + 32 * kB - 1) / (32 * kB), 0};
  t.count = t.m * t.n;
  const auto kernel = direct ? matmul8_split_kernel<T, kA, kB, true> : matmul8_split_kernel<T, kA, kB, false>;
  hipLaunchKernelGGL(kernel, dim3(t.count), dim3(256), 0, stream, p, t);
  return hipGetLastError();
}

template <uint32_t kG>
hipError_t launch_few(const Product& p, bool wide, bool direct, hipStream_t stream) {
  // workgroups of the same columns on one XCD, behind one L2
  const uint32_t across = (p.n + 127) / 128 * 8, wgs = across * ((p.m + 8 * kG - 1) / (8 * kG));
  // all workgroups at once if the CUs' LDS holds them, with as many wavefronts as it then has room for
  constexpr uint32_t each = kAhead<kG> * kStage<kG>, kLds = 160 << 10;
  const uint32_t share = kLds / std::min((wgs + kCus - 1) / kCus, 4u), stages = p.k / kDepth;
  const uint32_t waves = std::max(1u, std::min({kFewWaves<kG>, share / each, (stages + 1) / 2}));
  const auto kernel = direct ? matmul8_few_kernel<kG, true> : matmul8_few_kernel<kG, false>;
  hipLaunchKernelGGL(kernel, dim3(wgs), dim3(waves * 64), waves * each, stream, p, uint32_t(wide), across);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_few_groups(const Product& p, uint32_t groups, bool direct, hipStream_t stream) {
  constexpr bool wide = sizeof(T) == 4;
  if (groups == 1) return launch_few<1>(p, wide, direct, stream);
  if (groups == 2) return launch_few<2>(p, wide, direct, stream);
  if (groups == 3) return launch_few<3>(p, wide, direct, stream);
  if (groups == 4) return launch_few<4>(p, wide, direct, stream);
  if (groups <= 6) return launch_few<6>(p, wide, direct, stream);
  if (groups <= 8) return launch_few<8>(p, wide, direct, stream);
  return launch_few<10>(p, wide, direct, stream);
}

// What a CU reads into its LDS decides in most sizes.  Over a workgroup's life, start and end included, that is 29 bytes a
// clock (772 x 2048 x 11008), 28 (300 x 1280 x 8192), 23 (67 x 1280 x 8192), 21 to 22 (128 and 512 x 4096 x 4096): the
// kernel is the one whose workgroups together read the fewest rows to a CU, and among
// equals the one of the smallest tiles.  In us, with the kernel that it takes and with the one of
// the next larger tiles: 200 x 4096 x 4096 11.3 (64 x 64), 12.4; 96 x 11008 x 4096 19.6 (96 x 64), 20.0.
template <typename T>
hipError_t launch_block(const Product& p, hipStream_t stream) {
  const bool direct = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.w) | uintptr_t(p.xld) | uintptr_t(p.wld)) & 15) == 0;
  // the larger tiles' kernels have the distances of a tile's rows in 32 bits
  const bool near = p.xld <= 1 << 24 && p.wld <= 1 << 24;
  auto count = [&](uint64_t down, uint64_t across) { return (p.m + down - 1) / down * ((p.n + across - 1) / across); };
  auto rows = [&](uint64_t down, uint64_t across) { return (count(down, across) + kCus - 1) / kCus * (down + across); };
  // few rows to a workgroup: as many as leave one to each CU
  const uint32_t eighths = (p.m + 7) / 8, split = std::max(1u, std::min(eighths, kCus / ((p.n + 15) / 16)));
  const uint32_t groups = (eighths + split - 1) / split;
  enum Which { kFew, k32x64, k64x64, k96x64, k128x64, k96x96, k128x128, k256x256 } which = kFew;
  uint64_t best = groups <= 10 ? rows(8 * groups, 16) : UINT64_MAX;
  auto offer = [&](Which kernel, uint64_t down, uint64_t across) {
    const uint64_t r = rows(down, across);
    if (r < best) best = r, which = kernel;
  };
  offer(k32x64, 32, 64);
  offer(k64x64, 64, 64);
  offer(k96x64, 96, 64);
  offer(k128x64, 128, 64);
  offer(k96x96, 96, 96);
  if (near) {
    offer(k128x128, 128, 128);
    offer(k256x256, 256, 256);
  }
  switch (which) {
    case kFew: return launch_few_groups<T>(p, groups, direct, stream);
    case k32x64: return launch_split<T, 1, 2>(p, direct, stream);
    case k64x64: return launch_split<T, 2, 2>(p, direct, stream);
    case k96x64: return launch_split<T, 3, 2>(p, direct, stream);
    case k128x64: return launch_split<T, 4, 2>(p, direct, stream);
    case k96x96: return launch_split<T, 3, 3>(p, direct, stream);
    case k128x128:
      if (!direct) return launch_tiles<T, 2, 2, false>(p, stream);
      return count(128, 128) <= kCus ? launch_tiles<T, 2, 4, true>(p, stream) : launch_tiles<T, 2, 2, true>(p, stream);
    case k256x256: return direct ? launch_tiles<T, 4, 2, true>(p, stream) : launch_tiles<T, 4, 2, false>(p, stream);
  }
  return hipErrorInvalidValue;
}

// Blocks of the output that a launch takes: offsets within them, and workgroups, in 32 bits.
constexpr int64_t kMostRows = 1 << 19, kMostCols = 1 << 20;

template <typename T>
hipError_t launch_type(const etc_matmul8_args& a, hipStream_t stream) {
  for (int64_t i = 0; i < a.out.rows; i += kMostRows) {
    for (int64_t j = 0; j < a.out.cols; j += kMostCols) {
      const Mat8 x = mat8(a.x, i), w = mat8(a.w, j);
      const Product p{x.p, w.p, x.ld, w.ld, x.scale, w.scale, x.sld, w.sld, uint32_t(std::min(kMostRows, a.out.rows - i)),
                      uint32_t(std::min(kMostCols, a.out.cols - j)), uint32_t(a.x.cols), mat<T>(a.out, i).p + j, a.out.ld,
                      a.bias.data ? static_cast<const T*>(a.bias.data) + j : nullptr};
      const hipError_t e = launch_block<T>(p, stream);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_matmul8(const etc_matmul8_args& a, hipStream_t stream) {
  return a.out.dtype == ETC_DTYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace etc
