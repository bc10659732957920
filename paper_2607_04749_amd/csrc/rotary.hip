// rotary.hip -- rotary positions (etc_rotary).
//
//   a' = scale (a cos - b sin), b' = scale (b cos + a sin), the angle position * freq[pair]
//
// HBM bound: x is read and out written once.  Angles are worked out in turns and in
// 64 bits, where the whole turns are dropped; what is left has an error of 2^-26 of a turn
// (and, of t turns, t 2^-52).  No table of sines: a lane works its own out while the heads are on their way.
// 8192 tokens of 72 heads of 128 bf16 (302 MB): 50.1 us, 6.0 TB/s; with the sines worked out for each head 69.
// One token: 3.1 us, most of it the launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "eight.hpp"

namespace etc {

namespace {

struct Turns {
  double freq[ETC_ROTARY_PAIRS];  // turns a position
  float scale;
  float sign;  // -1 for the gradient
  uint32_t pairs, head_dim;
};

// Products and sums are fused where it is written, so that all kernels round alike.
__device__ __forceinline__ void angle(double position, double freq, float scale, float sign, float* c, float* s) {
  const float part = float(__builtin_fma(position, freq, -rint(position * freq)));
  sincospif(2.0f * part, s, c);
  *c *= scale;
  *s *= scale * sign;
}

__device__ __forceinline__ void turn(float a, float b, float c, float s, float* to_a, float* to_b) {
  *to_a = __builtin_fmaf(a, c, -(b * s));
  *to_b = __builtin_fmaf(b, c, a * s);
}

// A lane has two blocks of 16 bytes, half the pairs' columns apart, of kHeads heads of
// a token, so that their sines are worked out once.  kHalf: the columns of the one
// block are those of the other's pairs; else each block has pairs of its own.  Other lanes have
// two blocks of what is copied.  Neighbouring lanes have neighbouring blocks, and heads
// that follow on each other: heads of 80 columns, of which 64 turn, 28.7 us (8192 x 40 of them, bf16)
// where lanes had four heads in a row and two blocks side by side 40.3.
constexpr uint32_t kThreads = 256;

struct Blocks {
  uint32_t n;              // lanes with work
  uint32_t heads, slices;  // a lane has every `slices`th head
  uint32_t units;          // pairs of blocks in a head, of which the first `turned` turn
  uint32_t turned;
  uint32_t apart, past;    // columns from the one block to the other: of those that turn, of those that do not
  Divisor by_token, by_unit;  // lanes of a token, units of a head
};

// kWhole: all blocks are whole
template <typename T, bool kHalf, uint32_t kHeads, bool kWhole>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Turns t, Blocks g, Mat<const T> x, Ids positions, Mat<T> out) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  if (at >= g.n) return;
  const uint32_t i = g.by_token.div(at), in_token = at - i * g.by_token.d;
  const uint32_t slice = g.by_unit.div(in_token), unit = in_token - slice * g.by_unit.d;
  const bool turns = unit < g.turned;
  // the columns of the two blocks, the ends of the runs that they are of, and whether those are less than a block
  uint32_t ja, jb, ea, eb;
  bool shorter;
  if (turns) {
    ja = unit * kC;
    jb = ja + g.apart;
    ea = kHalf ? t.pairs : 2 * t.pairs;
    eb = 2 * t.pairs;
    shorter = ea < kC;
  } else {
    ja = 2 * t.pairs + (unit - g.turned) * kC;
    jb = ja + g.past;
    ea = eb = t.head_dim;
    shorter = t.head_dim - 2 * t.pairs < kC;
  }
  const uint32_t wa = block_width<kC>(ja, ea), wb = block_width<kC>(jb, eb);
  Raw<T, kC, kWhole> a[kHeads], b[kHeads];
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h) {
    const uint32_t head = h * g.slices + slice;
    if (head >= g.heads) break;
    const T* from = x.p + int64_t(i) * x.ld + int64_t(head) * t.head_dim;
    a[h].template load<true>(from + ja, wa, shorter);
    if (wb) b[h].template load<true>(from + jb, wb, shorter);
    else b[h].zero();
  }
  compiler_fence();
  float c[kC], s[kC];
  if (turns) {
    const double position = double(positions.at(i));
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) {
      const uint32_t pair = kHalf ? ja + e : e < kC / 2 ? ja / 2 + e : jb / 2 + e - kC / 2;
      angle(position, t.freq[min(pair, uint32_t(ETC_ROTARY_PAIRS - 1))], t.scale, t.sign, &c[e], &s[e]);
    }
  }
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h) {
    const uint32_t head = h * g.slices + slice;
    if (head >= g.heads) break;
    T* to = out.p + int64_t(i) * out.ld + int64_t(head) * t.head_dim;
    if (turns) {
      float u[kC], v[kC], p[kC], q[kC];
      a[h].widen(u, wa);
      b[h].widen(v, wb);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) {
        if (kHalf) {
          turn(u[e], v[e], c[e], s[e], &p[e], &q[e]);
        } else if (e % 2 == 0) {
          turn(u[e], u[e + 1], c[e / 2], s[e / 2], &p[e], &p[e + 1]);
          turn(v[e], v[e + 1], c[kC / 2 + e / 2], s[kC / 2 + e / 2], &q[e], &q[e + 1]);
        }
      }
      a[h].narrow(p);
      b[h].narrow(q);
    } else if (!kWhole) {  // as it is, from the block's beginning on
      float u[kC], v[kC];
      a[h].widen(u, wa);
      b[h].widen(v, wb);
      a[h].narrow(u);
      b[h].narrow(v);
    }
    // one store for all lanes of a line, those that turn and those that copy
    a[h].template store<kWhole>(to + ja, wa);
    if (wb) b[h].template store<kWhole>(to + jb, wb);
  }
}

template <typename T, bool kHalf>
hipError_t launch_layout(const etc_rotary_args& a, const Turns& t, hipStream_t stream) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t heads = uint32_t(a.x.cols / a.head_dim);
  const bool in_place = a.x.data == a.out.data;  // columns past the pairs are where they belong
  const uint32_t past = in_place ? 0 : t.head_dim - 2 * t.pairs;
  const bool whole = t.pairs % kC == 0 && past % kC == 0;
  const uint32_t blocks = kHalf ? 2 * blocks_per_row(t.pairs, kC) : blocks_per_row(2 * t.pairs, kC);
  const uint32_t turned = (blocks + 1) / 2, copied = (blocks_per_row(past, kC) + 1) / 2, units = turned + copied;
  // sines once for several heads, where that leaves lanes enough
  const uint32_t each = int64_t(a.x.rows) * heads * units >= (1 << 20) ? 4 : 1;
  const uint32_t slices = (heads + each - 1) / each, lanes = slices * units;  // of a token
  const int64_t most = std::max<int64_t>(1, INT32_MAX / lanes);
  for (int64_t at = 0; at < a.x.rows; at += most) {
    const uint32_t rows = uint32_t(std::min(most, a.x.rows - at));
    const uint32_t wide = a.positions.dtype == ETC_IDS_I64;
    const Ids ids{static_cast<const char*>(a.positions.data) + at * (wide ? 8 : 4), wide};
    const Blocks g{rows * lanes, heads, slices, units, turned, kHalf ? t.pairs : turned * kC, copied * kC, Divisor(lanes),
                   Divisor(units)};
    const auto kernel = whole ? each == 1 ? rotary_kernel<T, kHalf, 1, true> : rotary_kernel<T, kHalf, 4, true>
                              : each == 1 ? rotary_kernel<T, kHalf, 1, false> : rotary_kernel<T, kHalf, 4, false>;
    hipLaunchKernelGGL(kernel, dim3((g.n + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, t, g, cmat<T>(a.x, at), ids,
                       mat<T>(a.out, at));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_type(const etc_rotary_args& a, hipStream_t stream) {
  Turns t;
  const etc_rotary_desc& d = *a.rotary;
  for (int32_t j = 0; j < d.pairs; ++j) t.freq[j] = d.freq[j] * 0.15915494309189533577;  // 1 / 2 pi
  for (int32_t j = d.pairs; j < ETC_ROTARY_PAIRS; ++j) t.freq[j] = 0.0;
  t.scale = float(d.scale);
  t.sign = a.backward ? -1.0f : 1.0f;
  t.pairs = uint32_t(d.pairs);
  t.head_dim = uint32_t(a.head_dim);
  return d.layout == ETC_ROTARY_HALF ? launch_layout<T, true>(a, t, stream) : launch_layout<T, false>(a, t, stream);
}

}  // namespace

hipError_t launch_rotary(const etc_rotary_args& a, hipStream_t stream) {
  return a.x.dtype == ETC_DTYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace etc
