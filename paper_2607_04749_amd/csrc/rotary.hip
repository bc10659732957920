// rotary.hip -- rotary positions (etc_rotary) and their frequencies.
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

constexpr uint32_t kFlatThreads = 256;

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

// Any sizes: a lane has one pair, or one column past the pairs.
template <typename T, bool kHalf>
__global__ __launch_bounds__(kFlatThreads) void rotary_pair_kernel(Turns t, uint64_t n, uint32_t heads, uint32_t items,
                                                                   Mat<const T> x, Ids positions, Mat<T> out) {
  const uint64_t at = uint64_t(blockIdx.x) * kFlatThreads + threadIdx.x;
  if (at >= n) return;
  const uint32_t item = uint32_t(at % items);
  const uint64_t rest = at / items;
  const uint64_t i = rest / heads;
  const uint64_t head = uint64_t(rest - i * heads) * t.head_dim;
  const T* from = x.p + int64_t(i) * x.ld + head;
  T* to = out.p + int64_t(i) * out.ld + head;
  if (item >= t.pairs) {
    to[item + t.pairs] = from[item + t.pairs];
    return;
  }
  const uint32_t ja = kHalf ? item : 2 * item, jb = kHalf ? item + t.pairs : 2 * item + 1;
  float c, s;
  angle(double(positions.at(i)) * t.freq[item], t.scale, t.sign, &c, &s);
  const float a = float(from[ja]), b = float(from[jb]);
  to[ja] = T(a * c - b * s);
  to[jb] = T(b * c + a * s);
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
  const uint32_t heads = uint32_t(a.x.cols / a.head_dim);
  const bool in_place = a.x.data == a.out.data;  // columns past the pairs are where they belong
  const uint32_t items = in_place ? t.pairs : t.head_dim - t.pairs;
  const auto kernel = d.layout == ETC_ROTARY_HALF ? rotary_pair_kernel<T, true> : rotary_pair_kernel<T, false>;
  const int64_t most = std::max<int64_t>(1, INT32_MAX / (int64_t(heads) * items));
  for (int64_t at = 0; at < a.x.rows; at += most) {
    const int64_t rows = std::min(most, a.x.rows - at);
    const uint64_t n = uint64_t(rows) * heads * items;
    const uint32_t wide = a.positions.dtype == ETC_IDS_I64;
    const Ids ids{static_cast<const char*>(a.positions.data) + at * (wide ? 8 : 4), wide};
    hipLaunchKernelGGL(kernel, dim3(uint32_t((n + kFlatThreads - 1) / kFlatThreads)), dim3(kFlatThreads), 0, stream, t, n, heads,
                       items, cmat<T>(a.x, at), ids, mat<T>(a.out, at));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(const etc_rotary_args& a, hipStream_t stream) {
  return a.x.dtype == ETC_DTYPE_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

}  // namespace etc
