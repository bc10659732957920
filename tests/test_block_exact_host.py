"""The exact cases of the norm's weight gradient notice what they are for: a sum
that lacks a row, the rows of one wavefront or workgroup, or a row that is there
twice, is not the one expected in any column.  The mistakes are planted in the oracle."""
import numpy as np
import pytest

import block_exact


@pytest.mark.parametrize("case", block_exact.DWEIGHT, ids=str)
def test_any_rows_less_or_twice_are_another_sum(case):
    rows, cols, _, _, group = case
    grad, x, scale, r, _ = block_exact.dweight_case(case)
    right = block_exact.dweight_sums(grad, x, scale, group, r)
    at = np.arange(rows)
    for lost in (at == 0, at == rows // 2, at == rows - 1, at % 16 == rows % 16, at % 64 < 4, at // 4 % 256 == 0):
        if not lost.any():
            continue
        fewer, twice = r.copy(), r.copy()
        fewer[lost], twice[lost] = 0, 2 * r[lost]
        terms = block_exact.wide(x, scale, group) * grad
        for other in (fewer, twice):
            wrong = np.einsum("i,ij->j", other.astype(np.int64), terms.astype(np.int64))
            assert np.all(wrong != right)
