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

  // the eight 16-bit numbers of columns 8 * block .. 8 * block + 7 of row i, two to a word
  __host__ __device__ void bits(uint64_t i, uint32_t block, uint32_t (&w)[4]) const {
    const uint64_t r = row0 + i;
    w[0] = block;
    w[1] = uint32_t(r);
    w[2] = uint32_t(r >> 32);
    w[3] = call;
    philox4x32_10(w, k0, k1);
  }
  // v scaled where kept and 0 where dropped, whatever it is (a product with 0
  // would keep NaN); limit >= 1.  A number is in the upper half of a word for the
  // comparison: below the limit where the word is at most (limit << 16) - 1,
  // which for 65536 is any word, whatever the lower half holds.
  __device__ __forceinline__ void apply(const uint32_t (&w)[4], float (&v)[8]) const {
    const uint32_t top = (limit << 16) - 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (e % 2 ? w[e / 2] : w[e / 2] << 16) > top ? v[e] * scale : 0.0f;
  }
};

}  // namespace etc
