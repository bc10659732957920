// adam.hip -- a step of Adam with decoupled weight decay over a range of a
// rank's four state arenas (etc_adam), in one pass.
//
//   g = c grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   master -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + wd master);  param = bf16(master)
//
// HBM bound: 16 bytes read and 14 written per element, in eight streams.  With
// all 32 wave slots of a CU taken the streams' requests got in each other's way;
// large launches of one-wavefront workgroups reserve LDS (never touched) so that
// ten share a CU.  181 M elements, MI355X, in us: workgroups of 256 lanes 1001,
// with non-temporal accesses 949; one wavefront with 25 a CU 906, 19 881, 16 869,
// 12 842, 10 822 (6.6 TB/s), 8 833.  Ten a CU from 2.6 M elements on; graph replays, in us:
//   M elements    0.3   0.9   1.5   2.6   4.0   8.0    16    32    64   181
//   all slots     3.0   5.6   8.9  14.8  22.8  42.0  82.5   162   325   923
//   ten a CU      3.0   6.2   9.1  14.6  22.1  39.9  75.5   147   293   834
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kThreads = 64;
constexpr uint32_t kLdsBytes = 16384;            // a tenth of a CU's
constexpr uint32_t kCappedGrid = 4 * 10 * 256;   // workgroups of four rounds; fewer keep all slots

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct AdamArgs {
  AdamFactors f;
  bf16* param;
  float *master, *m, *v;
  const float *grad, *grad_scale;
  uint64_t first, end;  // the range
  uint64_t start;       // of the launch: the first unit's first element
};

// A lane steps the four elements of one 16-byte unit of the fp32 arenas, as far
// as they lie in the range.
constexpr uint32_t kUnit = 4;

__device__ __forceinline__ void adam_step(const AdamArgs& a, float c, float grad, float& w, float& m, float& v) {
  const float g = grad * c;
  m = a.f.beta1 * m + a.f.rest1 * g;
  v = a.f.beta2 * v + a.f.rest2 * (g * g);
  w -= a.f.step_size * m / (sqrtf(v * a.f.root) + a.f.eps) + a.f.decay * w;
}

__global__ __launch_bounds__(kThreads) void adam_kernel(AdamArgs a) {
  const uint64_t at = a.start + (uint64_t(blockIdx.x) * kThreads + threadIdx.x) * kUnit;
  if (at >= a.end) return;
  const float c = a.grad_scale ? *a.grad_scale : 1.0f;
  if (at >= a.first && at + kUnit <= a.end) {
    const f32x4 g = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.grad + at));
    f32x4 w = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.master + at));
    f32x4 m = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.m + at));
    f32x4 v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.v + at));
#pragma unroll
    for (uint32_t e = 0; e < kUnit; ++e) {
      float we = w[e], me = m[e], ve = v[e];
      adam_step(a, c, g[e], we, me, ve);
      w[e] = we, m[e] = me, v[e] = ve;
    }
    const bf16x4 p = __builtin_convertvector(w, bf16x4);
    __builtin_nontemporal_store(w, reinterpret_cast<f32x4*>(a.master + at));
    __builtin_nontemporal_store(m, reinterpret_cast<f32x4*>(a.m + at));
    __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(a.v + at));
    __builtin_nontemporal_store(p, reinterpret_cast<bf16x4*>(a.param + at));
    return;
  }
  for (uint64_t i = at < a.first ? a.first : at; i < at + kUnit && i < a.end; ++i) {
    float w = a.master[i], m = a.m[i], v = a.v[i];
    adam_step(a, c, a.grad[i], w, m, v);
    a.master[i] = w;
    a.m[i] = m;
    a.v[i] = v;
    a.param[i] = bf16(w);
  }
}

}  // namespace

hipError_t launch_adam(const etc_adam_args& x, const AdamFactors& factors, hipStream_t stream) {
  AdamArgs a{factors};
  a.param = static_cast<bf16*>(x.arena[0]);
  a.master = static_cast<float*>(x.arena[1]);
  a.m = static_cast<float*>(x.arena[2]);
  a.v = static_cast<float*>(x.arena[3]);
  a.grad = static_cast<const float*>(x.grad);
  a.grad_scale = static_cast<const float*>(x.grad_scale);
  a.first = x.first;
  a.end = x.first + x.count;
  constexpr uint64_t most = uint64_t(1) << 32;  // elements of a launch: 2^30 lanes
  for (a.start = x.first / kUnit * kUnit; a.start < a.end; a.start += most) {
    const uint64_t units = (std::min(a.end - a.start, most) + kUnit - 1) / kUnit;
    const uint32_t wgs = uint32_t((units + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(adam_kernel, dim3(wgs), dim3(kThreads), wgs >= kCappedGrid ? kLdsBytes : 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace etc
