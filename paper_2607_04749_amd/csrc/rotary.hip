// rotary.hip -- rotary positions (etc_rotary).
//
//   a' = scale (a cos - b sin), b' = scale (b cos + a sin), the angle position * freq[pair]
//
// HBM bound: x is read and out written once.  Angles are worked out in turns and in
// 64 bits, where the whole turns are dropped; what is left has an error of 2^-26 of a turn.
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

__device__ __forceinline__ void angle(double turns, float scale, float sign, float* c, float* s) {
  const float part = float(turns - rint(turns));
  sincospif(2.0f * part, s, c);
  *c *= scale;
  *s *= scale * sign;
}

// ---------------------------------------------------------------------------
// Heads whose parts that turn and that do not are whole blocks of 16 bytes: a lane has
// two blocks, whose columns are pairs (kHalf: of either half of the pairs; else
// neighbours), of kHeads heads of a token, so that their sines are worked out once; or
// two blocks of what is copied.

constexpr uint32_t kThreads = 256;

struct Blocks {
  uint32_t n;            // lanes with work
  uint32_t heads;
  uint32_t units;        // of a lane (pairs of blocks; pairs) in a head, of which the first `turned` turn
  uint32_t turned;
  Divisor by_token, by_unit;  // lanes of a token, units of a head
};

template <typename T, bool kHalf, uint32_t kHeads>
__global__ __launch_bounds__(kThreads) void rotary_block_kernel(Turns t, Blocks g, Mat<const T> x, Ids positions, Mat<T> out) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  if (at >= g.n) return;
  const uint32_t i = g.by_token.div(at), in_token = at - i * g.by_token.d;
  const uint32_t slice = g.by_unit.div(in_token), unit = in_token - slice * g.by_unit.d;
  const bool turns = unit < g.turned;
  uint32_t ja, jb;  // the columns of the two blocks
  if (turns) {
    ja = kHalf ? unit * kC : unit * 2 * kC;
    jb = kHalf ? ja + t.pairs : ja + kC;
  } else {
    ja = 2 * t.pairs + (unit - g.turned) * 2 * kC;
    jb = ja + kC;
  }
  const bool second = jb < t.head_dim;
  const uint32_t head0 = slice * kHeads;
  Raw<T, kC, true> a[kHeads], b[kHeads];
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h) {
    if (head0 + h >= g.heads) break;
    const T* from = x.p + int64_t(i) * x.ld + int64_t(head0 + h) * t.head_dim;
    a[h].template load<true>(from + ja, kC, false);
    if (second) b[h].template load<true>(from + jb, kC, false);
  }
  compiler_fence();
  float c[kC], s[kC];
  if (turns) {
    const double position = double(positions.at(i));
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) angle(position * t.freq[unit * kC + e], t.scale, t.sign, &c[e], &s[e]);
  }
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h) {
    if (head0 + h >= g.heads) break;
    T* to = out.p + int64_t(i) * out.ld + int64_t(head0 + h) * t.head_dim;
    if (turns) {
      float u[kC], v[kC], p[kC], q[kC];
      a[h].widen(u, kC);
      b[h].widen(v, kC);
#pragma unroll
      for (uint32_t e = 0; e < kC; ++e) {
        if (kHalf) {
          p[e] = u[e] * c[e] - v[e] * s[e];
          q[e] = v[e] * c[e] + u[e] * s[e];
        } else if (e % 2 == 0) {
          p[e] = u[e] * c[e / 2] - u[e + 1] * s[e / 2];
          p[e + 1] = u[e + 1] * c[e / 2] + u[e] * s[e / 2];
          q[e] = v[e] * c[kC / 2 + e / 2] - v[e + 1] * s[kC / 2 + e / 2];
          q[e + 1] = v[e + 1] * c[kC / 2 + e / 2] + v[e] * s[kC / 2 + e / 2];
        }
      }
      a[h].narrow(p);
      b[h].narrow(q);
    }
    a[h].template store<true>(to + ja, kC);
    if (second) b[h].template store<true>(to + jb, kC);
  }
}

// Any other sizes: a lane has a pair, or a column past the pairs, of kHeads heads of a token.
template <typename T, bool kHalf, uint32_t kHeads>
__global__ __launch_bounds__(kThreads) void rotary_pair_kernel(Turns t, Blocks g, Mat<const T> x, Ids positions, Mat<T> out) {
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  if (at >= g.n) return;
  const uint32_t i = g.by_token.div(at), in_token = at - i * g.by_token.d;
  const uint32_t slice = g.by_unit.div(in_token), item = in_token - slice * g.by_unit.d;
  const bool turns = item < g.turned;
  const uint32_t ja = turns && !kHalf ? 2 * item : turns ? item : item + t.pairs, jb = kHalf ? item + t.pairs : 2 * item + 1;
  const uint32_t head0 = slice * kHeads;
  T a[kHeads], b[kHeads];
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h) {
    if (head0 + h >= g.heads) break;
    const T* from = x.p + int64_t(i) * x.ld + int64_t(head0 + h) * t.head_dim;
    a[h] = from[ja];
    if (turns) b[h] = from[jb];
  }
  compiler_fence();
  float c = 1.0f, s = 0.0f;
  if (turns) angle(double(positions.at(i)) * t.freq[item], t.scale, t.sign, &c, &s);
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h) {
    if (head0 + h >= g.heads) break;
    T* to = out.p + int64_t(i) * out.ld + int64_t(head0 + h) * t.head_dim;
    if (turns) {
      const float u = float(a[h]), v = float(b[h]);
      to[ja] = T(u * c - v * s);
      to[jb] = T(v * c + u * s);
    } else {
      to[ja] = a[h];
    }
  }
}

template <typename T, bool kHalf>
hipError_t launch_layout(const etc_rotary_args& a, const Turns& t, hipStream_t stream) {
  constexpr uint32_t kC = kLaneCols<T>;
  const uint32_t heads = uint32_t(a.x.cols / a.head_dim);
  const bool in_place = a.x.data == a.out.data;  // columns past the pairs are where they belong
  const bool blocks = t.pairs % kC == 0 && t.head_dim % kC == 0;
  const uint32_t past = in_place ? 0 : t.head_dim - 2 * t.pairs;
  const uint32_t items = blocks ? t.pairs / kC + (past / kC + 1) / 2 : t.pairs + past;  // lanes of a head
  // sines once for several heads, where that leaves lanes enough
  const uint32_t each = int64_t(a.x.rows) * heads * items >= (1 << 20) ? 4 : 1;
  const uint32_t lanes = (heads + each - 1) / each * items;  // of a token
  const int64_t most = std::max<int64_t>(1, INT32_MAX / lanes);
  for (int64_t at = 0; at < a.x.rows; at += most) {
    const uint32_t rows = uint32_t(std::min(most, a.x.rows - at));
    const uint32_t wide = a.positions.dtype == ETC_IDS_I64;
    const Ids ids{static_cast<const char*>(a.positions.data) + at * (wide ? 8 : 4), wide};
    const uint32_t n = rows * lanes;
    const dim3 wgs((n + kThreads - 1) / kThreads), threads(kThreads);
    const Blocks g{n, heads, items, blocks ? t.pairs / kC : t.pairs, Divisor(lanes), Divisor(items)};
    const auto kernel = blocks ? each == 1 ? rotary_block_kernel<T, kHalf, 1> : rotary_block_kernel<T, kHalf, 4>
                               : each == 1 ? rotary_pair_kernel<T, kHalf, 1> : rotary_pair_kernel<T, kHalf, 4>;
    hipLaunchKernelGGL(kernel, wgs, threads, 0, stream, t, g, cmat<T>(a.x, at), ids, mat<T>(a.out, at));
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
