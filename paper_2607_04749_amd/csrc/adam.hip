// adam.hip -- a step of Adam with decoupled weight decay over a range of a
// rank's four state arenas (etc_adam), in one pass.
//
//   g = c grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   master -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + wd master);  param = bf16(master)
//
// HBM bound: 16 bytes read and 14 written per element.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ops.hpp"

namespace etc {

namespace {

constexpr uint32_t kThreads = 256;

struct AdamArgs {
  bf16* param;
  float *master, *m, *v;
  const float *grad, *grad_scale;
  uint64_t n;
  float beta1, rest1, beta2, rest2;  // rest = 1 - beta, from 64 bits
  float step_size;                   // lr / (1 - beta1^t)
  float root;                        // 1 / (1 - beta2^t)
  float eps, decay;                  // decay = lr * weight_decay
};

__global__ __launch_bounds__(kThreads) void adam_kernel(AdamArgs a) {
  const float c = a.grad_scale ? *a.grad_scale : 1.0f;
  for (uint64_t i = uint64_t(blockIdx.x) * kThreads + threadIdx.x; i < a.n; i += uint64_t(gridDim.x) * kThreads) {
    const float g = a.grad[i] * c, w = a.master[i];
    const float m = a.beta1 * a.m[i] + a.rest1 * g;
    const float v = a.beta2 * a.v[i] + a.rest2 * (g * g);
    const float x = w - (a.step_size * m / (sqrtf(v * a.root) + a.eps) + a.decay * w);
    a.m[i] = m;
    a.v[i] = v;
    a.master[i] = x;
    a.param[i] = bf16(x);
  }
}

}  // namespace

hipError_t launch_adam(const etc_adam_args& x, hipStream_t stream) {
  AdamArgs a{};
  a.param = static_cast<bf16*>(x.arena[0]) + x.first;
  a.master = static_cast<float*>(x.arena[1]) + x.first;
  a.m = static_cast<float*>(x.arena[2]) + x.first;
  a.v = static_cast<float*>(x.arena[3]) + x.first;
  a.grad = static_cast<const float*>(x.grad) + x.first;
  a.grad_scale = static_cast<const float*>(x.grad_scale);
  a.n = x.count;
  a.beta1 = float(x.beta1);
  a.rest1 = float(1.0 - x.beta1);
  a.beta2 = float(x.beta2);
  a.rest2 = float(1.0 - x.beta2);
  a.step_size = float(x.lr / (1.0 - std::pow(x.beta1, double(x.step))));
  a.root = float(1.0 / (1.0 - std::pow(x.beta2, double(x.step))));
  a.eps = float(x.eps);
  a.decay = float(x.lr * x.weight_decay);
  const uint64_t wgs = std::min<uint64_t>((x.count + kThreads - 1) / kThreads, 65536);
  hipLaunchKernelGGL(adam_kernel, dim3(uint32_t(wgs)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace etc
