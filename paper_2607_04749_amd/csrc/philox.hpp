// philox.hpp -- the random bits of dropout: Philox4x32-10, the counter-based
// generator of Salmon, Moraes, Dror and Shaw, "Parallel Random Numbers: As
// Easy as 1, 2, 3" (SC 2011): ten rounds of two 32 x 32 -> 64 bit products,
// keyed by a Weyl sequence.  One call gives four words from a counter and a
// key alone, so any part of a mask can be found anywhere, without state.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace etc {

// a ^ b ^ c, in one instruction where there is one
__host__ __device__ inline uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
#else
  return a ^ b ^ c;
#endif
}

__host__ __device__ inline void philox4x32_10(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t a = uint64_t(0xD2511F53u) * c[0], b = uint64_t(0xCD9E8D57u) * c[2];
    c[0] = xor3(uint32_t(b >> 32), c[1], k0);
    c[2] = xor3(uint32_t(a >> 32), c[3], k1);
    c[1] = uint32_t(b);
    c[3] = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// A dropout, as kernels take it: element (i, j) is dropped where its 16 bits
// are below `limit` (0: none, 65536: all).
struct Drop {
  uint32_t k0, k1, call, limit;
  uint64_t row0;
  float scale;  // of what is kept: 65536 / (65536 - limit)

  // The 16-bit numbers of columns col .. col + kC - 1 (a multiple of kC) of row i, two to a word.
  template <uint32_t kC>
  __host__ __device__ void bits(uint64_t i, uint64_t col, uint32_t (&w)[kC / 2]) const {
    const uint64_t r = row0 + i;
    uint32_t c[4] = {uint32_t(col / 8), uint32_t(r), uint32_t(r >> 32), call};
    philox4x32_10(c, k0, k1);
    const uint32_t c0 = c[0], c1 = c[1], c2 = c[2], c3 = c[3];
    if constexpr (kC == 8) {
      w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
    } else {
      w[0] = col & 4 ? c2 : c0;
      w[1] = col & 4 ? c3 : c1;
    }
  }
  // v scaled where kept and 0 where dropped, whatever it is (a product with 0
  // would keep NaN); limit >= 1.  A number is in the upper half of a word for the
  // comparison: below the limit where the word is at most (limit << 16) - 1,
  // which for 65536 is any word, whatever the lower half holds.
  template <uint32_t kC>
  __device__ __forceinline__ void apply(const uint32_t (&w)[kC / 2], float (&v)[kC]) const {
    const uint32_t top = (limit << 16) - 1;
#pragma unroll
    for (uint32_t e = 0; e < kC; ++e) v[e] = (e % 2 ? w[e / 2] : w[e / 2] << 16) > top ? v[e] * scale : 0.0f;
  }
};

}  // namespace etc
