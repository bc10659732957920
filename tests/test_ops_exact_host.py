"""The exact cases of the operators' sums notice what they are for: a sum that
lacks one token or one row, or that has one twice, is not the one expected.  The
mistakes are planted in the oracle."""
import numpy as np
import pytest

import op_exact


@pytest.mark.parametrize("case", [c for c in op_exact.GRAD if c[0] * c[1] < 1 << 22], ids=str)
def test_one_token_more_or_less_is_another_gradient(case):
    v, g, before, drop = op_exact.grad_case(case)
    right, added = op_exact.grad_sums(v, g, before, drop)
    inside = np.flatnonzero((v >= 0) & (v < before.shape[0]))
    kept = np.broadcast_to(op_exact._kept(*g.shape, drop), g.shape)
    for at in (inside[0], inside[inside.size // 2], inside[-1]):
        fewer = v.copy()
        fewer[at] = -1
        wrong, wrong_added = op_exact.grad_sums(fewer, g, before, drop)
        changed = wrong != right
        assert np.array_equal(changed[v[at]], kept[at] != 0) and changed.sum() == (kept[at] != 0).sum()
        assert np.array_equal(wrong_added != added, changed)
        twice = g.copy()
        twice[at] *= 2
        assert np.array_equal(op_exact.grad_sums(v, twice, before, drop)[0] != right, changed)


@pytest.mark.parametrize("case", [c for c in op_exact.BIAS if c[0] * c[1] < 1 << 22], ids=str)
def test_one_row_less_is_another_sum(case):
    g, before, drop = op_exact.bias_case(case)
    dropped, right, added = op_exact.bias_sums(g, before, drop)
    for at in (0, g.shape[0] // 2, g.shape[0] - 1):
        fewer = g.copy()
        fewer[at] = 0
        _, wrong, wrong_added = op_exact.bias_sums(fewer, before, drop)
        assert np.array_equal(wrong != right, dropped[at] != 0) and np.array_equal(wrong_added != added, dropped[at] != 0)
