// opshost.cpp -- host side of the operators' helpers, built and run by
// tests/test_ops_host.py: dropout's generator, the division by a product, the
// cut of a matrix into launches, and the layout of the argument structs.
// Test code: it prints what it finds; the test holds what is expected.
#include <cstddef>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "ops.hpp"

static void layout() {
#define AT(T, f) printf(#T "." #f " %zu\n", offsetof(T, f))
#define SIZE(T) printf(#T " %zu\n", sizeof(T))
  SIZE(etc_matrix); SIZE(etc_ids); SIZE(etc_dropout_desc);
  AT(etc_embed_args, table); AT(etc_embed_args, drop); AT(etc_embed_args, row0); SIZE(etc_embed_args);
  AT(etc_embed_grad_args, grad); AT(etc_embed_grad_args, drop); AT(etc_embed_grad_args, workspace);
  AT(etc_embed_grad_args, accumulate); SIZE(etc_embed_grad_args);
  AT(etc_dropout_args, out); AT(etc_dropout_args, drop); SIZE(etc_dropout_args);
  AT(etc_dropout_grad_args, drop); AT(etc_dropout_grad_args, accumulate); SIZE(etc_dropout_grad_args);
  AT(etc_adam_args, grad_scale); AT(etc_adam_args, first); AT(etc_adam_args, lr); AT(etc_adam_args, step); SIZE(etc_adam_args);
}

int main(int argc, char** argv) {
  if (argc < 2) return 2;
  if (!strcmp(argv[1], "layout")) {
    layout();
  } else if (!strcmp(argv[1], "philox") && argc == 8) {
    uint32_t c[4];
    for (int i = 0; i < 4; ++i) c[i] = uint32_t(strtoul(argv[2 + i], nullptr, 16));
    etc::philox4x32_10(c, uint32_t(strtoul(argv[6], nullptr, 16)), uint32_t(strtoul(argv[7], nullptr, 16)));
    printf("%08x %08x %08x %08x\n", c[0], c[1], c[2], c[3]);
  } else if (!strcmp(argv[1], "divide")) {
    uint64_t bad = 0, seed = 12345;
    for (uint32_t k = 0; k < 200000; ++k) {
      seed = seed * 6364136223846793005ull + 1442695040888963407ull;
      const uint32_t d = k < 4096 ? k + 1 : uint32_t(seed >> 36) % ((1u << (1 + k % 28))) + 1;
      const etc::Divisor by(d);
      const uint32_t n0 = uint32_t(seed >> 33), q0 = n0 / d;
      for (uint32_t n : {0u, 1u, d - 1, d, n0, q0 * d, q0 * d ? q0 * d - 1 : 0, 0x7FFFFFFFu})
        if (n <= 0x7FFFFFFFu && by.div(n) != n / d) ++bad;
    }
    printf("%llu\n", (unsigned long long)bad);
  } else if (!strcmp(argv[1], "runs") && argc == 6) {
    const int64_t rows = atoll(argv[2]), cols = atoll(argv[3]);
    (void)etc::for_row_runs(rows, cols, uint32_t(atoi(argv[4])), uint32_t(atoi(argv[5])), [&](int64_t first, const etc::BlockGrid& g) -> hipError_t {
      printf("%lld %u %u %u %u\n", (long long)first, g.n, g.rows, g.cols, g.per_row.d);
      return hipSuccess;
    });
  }
  return 0;
}
