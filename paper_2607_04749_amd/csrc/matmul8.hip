// matmul8.hip -- products of 8-bit integers with a scale for each row of either
// operand (etc_matmul8).
//
//   out[m, n] = sx[m] sw[n] (sum over k of x[m, k] w[n, k]) + bias[n]
//
// The sums are exact in 32-bit integers, so how they are split changes no bit.
#include <hip/hip_runtime.h>

#include <algorithm>

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
};

// Four neighbouring columns n .. n + 3 of row m, as far as there are any.
template <typename T>
__device__ __forceinline__ void store4(const Product& p, uint32_t m, uint64_t n, const int* sums, float x_scale) {
  const uint32_t width = n >= p.n ? 0 : uint32_t(min(uint64_t(4), p.n - n));
  float v[4];
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e) {
    if (e >= width) break;
    v[e] = float(sums[e]) * x_scale * p.w_scale(uint32_t(n) + e);
    if (p.bias) v[e] += float(static_cast<const T*>(p.bias)[n + e]);
  }
  T* out = static_cast<T*>(p.out) + int64_t(m) * p.ld + int64_t(n);
  Raw<T, 4, false> raw;
  raw.narrow(v);
  if (width) raw.store(out, width);
}

// ---------------------------------------------------------------------------
// Few rows: the weights are read once, and everything waits for them.  A workgroup
// has 16 columns of the output and all its rows (kM blocks of 16); its wavefronts
// share the sums' length between them, each with its operands straight from memory into
// registers, and add up in LDS.

constexpr uint32_t kFewStep = 64;  // of the sum by one matrix instruction
constexpr uint32_t kFewBatch = 4;  // steps whose loads are under way at once

template <uint32_t kM>
__device__ __forceinline__ void few_multiply(const i32x4& w, const i32x4 (&x)[kM], i32x4 (&acc)[kM]) {
#pragma unroll
  for (uint32_t t = 0; t < kM; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x[t], acc[t], 0, 0, 0);
}

__device__ __forceinline__ i32x4 load16(const uint8_t* p) {
  Raw8<16, true> r;
  r.load(p, 16, false);
  return i32x4{int(r.w[0]), int(r.w[1]), int(r.w[2]), int(r.w[3])};
}

__device__ __forceinline__ i32x4 load16_tail(const uint8_t* p, uint64_t k, uint32_t end) {
  Raw8<16, false> r;
  r.zero();
  const uint32_t width = block_width<16>(k, end);
  if (width) r.load(p + k, width, end < 16);
  r.shift(width);
  return i32x4{int(r.w[0]), int(r.w[1]), int(r.w[2]), int(r.w[3])};
}

template <typename T, uint32_t kM>
__global__ __launch_bounds__(1024) void matmul8_few_kernel(Product p) {
  extern __shared__ i32x4 parts[];  // [wavefront][kM][lane]
  const uint32_t lane = threadIdx.x % 64, waves = blockDim.x / 64;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint64_t n0 = uint64_t(blockIdx.x) * 16;
  // rows past the end repeat the last one; what comes of them is not stored
  const uint8_t* w = p.w + int64_t(min(n0 + lane % 16, uint64_t(p.n) - 1)) * p.wld;
  const uint8_t* x[kM];
#pragma unroll
  for (uint32_t t = 0; t < kM; ++t) x[t] = p.x + int64_t(min(t * 16 + lane % 16, p.m - 1)) * p.xld;
  const uint32_t steps = p.k / kFewStep, part = lane / 16 * 16;
  const uint32_t from = uint32_t(uint64_t(steps) * wave / waves), to = uint32_t(uint64_t(steps) * (wave + 1) / waves);
  i32x4 acc[kM] = {};
  uint32_t s = from;
  for (; s + kFewBatch <= to; s += kFewBatch) {
    i32x4 rw[kFewBatch], rx[kFewBatch][kM];
#pragma unroll
    for (uint32_t b = 0; b < kFewBatch; ++b) {
      const uint64_t k = uint64_t(s + b) * kFewStep + part;
      rw[b] = load16(w + k);
#pragma unroll
      for (uint32_t t = 0; t < kM; ++t) rx[b][t] = load16(x[t] + k);
    }
    compiler_fence();
#pragma unroll
    for (uint32_t b = 0; b < kFewBatch; ++b) few_multiply<kM>(rw[b], rx[b], acc);
  }
  for (; s < to; ++s) {
    const uint64_t k = uint64_t(s) * kFewStep + part;
    i32x4 rx[kM];
#pragma unroll
    for (uint32_t t = 0; t < kM; ++t) rx[t] = load16(x[t] + k);
    few_multiply<kM>(load16(w + k), rx, acc);
  }
  if (wave == waves - 1 && p.k % kFewStep) {
    const uint64_t k = uint64_t(steps) * kFewStep + part;
    i32x4 rx[kM];
#pragma unroll
    for (uint32_t t = 0; t < kM; ++t) rx[t] = load16_tail(x[t], k, p.k);
    few_multiply<kM>(load16_tail(w, k, p.k), rx, acc);
  }
#pragma unroll
  for (uint32_t t = 0; t < kM; ++t) parts[(wave * kM + t) * 64 + lane] = acc[t];
  __syncthreads();
  for (uint32_t at = threadIdx.x; at < kM * 64; at += blockDim.x) {
    i32x4 sum = parts[at];
    for (uint32_t v = 1; v < waves; ++v) sum += parts[v * kM * 64 + at];
    const uint32_t m = at / 64 * 16 + at % 16;
    if (m >= p.m) continue;
    const int sums[4] = {sum[0], sum[1], sum[2], sum[3]};
    store4<T>(p, m, n0 + at % 64 / 16 * 4, sums, p.x_scale(m));
  }
}

// ---------------------------------------------------------------------------
// Tiles of 64 kF x 64 kF of the output by four wavefronts, each of which has a
// quarter in registers.  128 columns of the operands at a time stand in LDS, twice:
// while one copy is multiplied the other one is filled, straight from memory
// (kDirect: rows at multiples of 16 bytes), or by way of registers.

constexpr uint32_t kDepth = 128;

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

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

template <typename T, uint32_t kF, bool kDirect>
__global__ __launch_bounds__(256, kF == 4 ? 1 : 2) void matmul8_tile_kernel(Product p, Tiles tiles) {
  constexpr uint32_t kTile = 64 * kF;
  constexpr uint32_t kLoads = kTile / 32;  // of a wavefront, of 8 rows each, for one operand
  constexpr uint32_t kOperand = kTile * kDepth, kCopy = 2 * kOperand;
  __shared__ __attribute__((aligned(1024))) uint8_t buffer[2 * kCopy];  // copies of x's and w's rows
  uint32_t tm, tn;
  place_tile(tiles, &tm, &tn);
  const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint64_t m0 = uint64_t(tm) * kTile, n0 = uint64_t(tn) * kTile;
  const uint8_t* base[2] = {p.x + int64_t(m0) * p.xld, p.w + int64_t(n0) * p.wld};
  // Row r of a tile has its chunk c of 16 bytes at place c ^ (r % 8), so that reads of 8 rows
  // of one chunk touch all banks; a load's lanes have the chunks that fill 8 rows in order.
  const uint32_t chunk = (lane % 8 ^ lane / 8) * 16;
  uint32_t offset[2][kLoads];
#pragma unroll
  for (uint32_t i = 0; i < kLoads; ++i) {
    const uint32_t row = (wave * kLoads + i) * 8 + lane / 8;  // rows past the end repeat the last one
    offset[0][i] = uint32_t(min(uint64_t(row), p.m - 1 - m0)) * uint32_t(p.xld) + chunk;
    offset[1][i] = uint32_t(min(uint64_t(row), p.n - 1 - n0)) * uint32_t(p.wld) + chunk;
  }
  Raw8<16, false> staged[2][kLoads];
  // load `i` of operand o, of 128 columns from k on, into copy c or on its way there in registers
  auto start = [&](uint64_t k, uint32_t c, uint32_t o, uint32_t i) {
    if constexpr (kDirect)
      __builtin_amdgcn_global_load_lds((global_void*)(base[o] + k + offset[o][i]),
                                       (lds_void*)&buffer[c * kCopy + o * kOperand + (wave * kLoads + i) * 1024], 16, 0, 0);
    else staged[o][i].load(base[o] + k + offset[o][i], 16, false);
  };
  auto place = [&](uint32_t c) {
#pragma unroll
    for (uint32_t o = 0; o < 2; ++o) {
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i) {
        const Raw8<16, false>& r = staged[o][i];
        *reinterpret_cast<i32x4*>(&buffer[c * kCopy + o * kOperand + (wave * kLoads + i) * 1024 + lane * 16]) =
            i32x4{int(r.w[0]), int(r.w[1]), int(r.w[2]), int(r.w[3])};
      }
    }
  };
  // until all wavefronts have filled their part of a copy
  auto finish = [&](uint32_t c) {
    if (!kDirect) place(c);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };

  const uint32_t left[2] = {wave % 2 * (kTile / 2), wave / 2 * (kTile / 2)};  // the wavefront's rows of x and of w
  uint32_t place0[2];  // of a lane's operand in the first step; in step s, s * 32 is added to its chunk's place
#pragma unroll
  for (uint32_t o = 0; o < 2; ++o) place0[o] = o * kOperand + (left[o] + lane % 32) * kDepth + (lane / 32 ^ lane % 8) * 16;
  auto read = [&](uint32_t c, uint32_t step, uint32_t o, uint32_t b) {
    return *reinterpret_cast<const i32x4*>(&buffer[c * kCopy + (place0[o] ^ step * 32) + b * 32 * kDepth]);
  };

  i32x16 acc[kF][kF] = {};  // [of w][of x]
  i32x4 x[2][kF], w[2][kF];
  // Multiplies copy c, whose first operands are in x[0] and w[0].  `more`: meanwhile fills the other copy with the
  // columns from k on, and leaves its first operands in their place.  The order is kept as it
  // stands: reads of the next step's operands and loads of the next copy's, one by one between matrix instructions.
  auto multiply = [&](uint32_t c, bool more, uint64_t k) {
    constexpr uint32_t kEach = kF * kF, kReads = 2 * kF;
#pragma unroll
    for (uint32_t step = 0; step < 4; ++step) {
      const uint32_t now = step % 2, next = 1 - now;
#pragma unroll
      for (uint32_t q = 0; q < kEach; ++q) {
        if (more && step == 0) {
#pragma unroll
          for (uint32_t d = q * 2 * kLoads / kEach; d < (q + 1) * 2 * kLoads / kEach; ++d) start(k, 1 - c, d / kLoads, d % kLoads);
        }
        if (more && step == 3 && q == kEach / 2) finish(1 - c);
        __builtin_amdgcn_sched_barrier(0);
        acc[q / kF][q % kF] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[now][q / kF], x[now][q % kF], acc[q / kF][q % kF], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t r = 0; r < kReads; ++r) {
          const uint32_t b = r / 2, o = 1 - r % 2;
          i32x4& to = o ? w[next][b] : x[next][b];
          if (step < 3 && r * kEach * 3 / (4 * kReads) == q) to = read(c, step + 1, o, b);
          if (more && step == 3 && kEach / 2 + r * (kEach - kEach / 2) * 3 / (4 * kReads) == q) to = read(1 - c, 0, o, b);
        }
      }
    }
  };

  // The columns past whole stages come first, so that the loop has whole ones only.
  const uint32_t whole = p.k / kDepth, rest = p.k % kDepth;
  if (p.k) {
    if (rest) {
      const uint64_t k = uint64_t(whole) * kDepth;
      const uint32_t width = block_width<16>(k + chunk, p.k);
#pragma unroll
      for (uint32_t o = 0; o < 2; ++o) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) {
          staged[o][i].zero();
          if (width) staged[o][i].load(base[o] + k + offset[o][i], width, p.k < 16);
          staged[o][i].shift(width);
        }
      }
      if (kDirect) place(0);
    } else {
#pragma unroll
      for (uint32_t o = 0; o < 2; ++o) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) start(0, 0, o, i);
      }
    }
    finish(0);
#pragma unroll
    for (uint32_t b = 0; b < kF; ++b) x[0][b] = read(0, 0, 0, b), w[0][b] = read(0, 0, 1, b);
    uint32_t c = 0;
    for (uint32_t s = rest ? 0 : 1; s < whole; ++s) {
      multiply(c, true, uint64_t(s) * kDepth);
      c = 1 - c;
    }
    multiply(c, false, 0);
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
      bias[i][e] = p.bias ? float(static_cast<const T*>(p.bias)[n]) : 0.0f;
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
          v[e] = float(acc[i][j][4 * q + e]) * scale_x * scale_w[i][4 * q + e] + bias[i][4 * q + e];
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

template <typename T, uint32_t kF, bool kDirect>
hipError_t launch_tiles(const Product& p, hipStream_t stream) {
  constexpr uint32_t kTile = 64 * kF;
  Tiles t{(p.m + kTile - 1) / kTile, (p.n + kTile - 1) / kTile, 0};
  t.count = t.m * t.n;
  hipLaunchKernelGGL((matmul8_tile_kernel<T, kF, kDirect>), dim3(t.count), dim3(256), 0, stream, p, t);
  return hipGetLastError();
}

template <typename T, uint32_t kM>
hipError_t launch_few(const Product& p, hipStream_t stream) {
  const uint32_t wgs = (p.n + 15) / 16;
  // 64 KB of LDS at most
  const uint32_t waves = std::max(1u, std::min({wgs >= 512 ? 8u : 16u, 64 / kM, p.k / kFewStep}));
  hipLaunchKernelGGL((matmul8_few_kernel<T, kM>), dim3(wgs), dim3(waves * 64), waves * kM * 1024, stream, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_block(const Product& p, hipStream_t stream) {
  switch ((p.m + 15) / 16) {
    case 1: return launch_few<T, 1>(p, stream);
    case 2: return launch_few<T, 2>(p, stream);
    case 3: return launch_few<T, 3>(p, stream);
    case 4: return launch_few<T, 4>(p, stream);
    case 5: return launch_few<T, 5>(p, stream);
    case 6: return launch_few<T, 6>(p, stream);
    case 7: return launch_few<T, 7>(p, stream);
    case 8: return launch_few<T, 8>(p, stream);
  }
  const bool direct = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.w) | uintptr_t(p.xld) | uintptr_t(p.wld)) & 15) == 0;
  auto tiles = [&](uint64_t tile) { return ((p.m + tile - 1) / tile) * ((p.n + tile - 1) / tile); };
  if (tiles(256) >= 256) return direct ? launch_tiles<T, 4, true>(p, stream) : launch_tiles<T, 4, false>(p, stream);
  if (tiles(128) >= 256) return direct ? launch_tiles<T, 2, true>(p, stream) : launch_tiles<T, 2, false>(p, stream);
  return direct ? launch_tiles<T, 1, true>(p, stream) : launch_tiles<T, 1, false>(p, stream);
}

// Blocks of the output that a launch takes: offsets within them, and workgroups, in 32 bits.
constexpr int64_t kMostRows = 1 << 20, kMostCols = 1 << 20;

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
