// layout.cpp -- prints where the fields of the argument structs of the operators
// around a block's projections lie; built and run by tests/test_block_host.py.
#include <cstddef>
#include <cstdio>

#include "etc.h"

int main() {
#define AT(T, f) printf(#T "." #f " %zu\n", offsetof(T, f))
#define SIZE(T) printf(#T " %zu\n", sizeof(T))
  SIZE(etc_matrix8); AT(etc_matrix8, scale); AT(etc_matrix8, rows); AT(etc_matrix8, scale_ld); AT(etc_matrix8, group);
  SIZE(etc_norm_args); AT(etc_norm_args, weight); AT(etc_norm_args, out8); AT(etc_norm_args, rstd); AT(etc_norm_args, eps);
  SIZE(etc_norm_grad_args); AT(etc_norm_grad_args, x8); AT(etc_norm_grad_args, dweight); AT(etc_norm_grad_args, rstd);
  AT(etc_norm_grad_args, workspace_bytes); AT(etc_norm_grad_args, accumulate);
  SIZE(etc_store8_args); AT(etc_store8_args, col_scale); AT(etc_store8_args, out);
  SIZE(etc_load8_args); AT(etc_load8_args, out);
  SIZE(etc_matmul8_args); AT(etc_matmul8_args, w); AT(etc_matmul8_args, bias); AT(etc_matmul8_args, out);
  SIZE(etc_rotary_desc); AT(etc_rotary_desc, scale); AT(etc_rotary_desc, pairs); AT(etc_rotary_desc, layout);
  SIZE(etc_rotary_args); AT(etc_rotary_args, positions); AT(etc_rotary_args, rotary); AT(etc_rotary_args, head_dim);
  AT(etc_rotary_args, backward);
  return 0;
}
