"""The operators around a block's projections at the ends of what they take, without
a GPU."""
import copy
import ctypes
import pickle

import pytest

from paper_2607_04749_amd import etc
from test_block_host import E4M3, I8, mat8, norm_grad
from test_ops_host import F32, INVALID, NONE, OK, mat


@pytest.mark.parametrize("dtype", (I8, E4M3))
@pytest.mark.parametrize("group", (0, 32))
def test_kept_activations_of_no_elements(dtype, group):
    """The backward of a batch without tokens: no work, whether its input was kept in 8 bits or not.  What is given
    has to fit all the same."""
    for t in (etc.DTYPE_BF16, F32):
        e, e8 = mat(0, 16, t, ptr=0), mat8(0, 16, dtype, group, ptr=0, scale=0)
        w = mat(1, 16, t)
        assert norm_grad(grad=e, x=NONE, x8=e8, dx=e, weight=w, rstd=0) == OK, etc.last_error()
        assert norm_grad(grad=e, x=NONE, x8=e8, dx=e, weight=w, rstd=0, dweight=mat(1, 16, F32), accumulate=1) == OK
        assert norm_grad(grad=e, x=NONE, x8=mat8(0, 8, dtype, group, ptr=0, scale=0), dx=e, weight=w, rstd=0) == INVALID
        assert norm_grad(grad=e, x=NONE, x8=mat8(3, 16, dtype, group, ptr=0, scale=0), dx=e, weight=w, rstd=0) == INVALID
        assert norm_grad(grad=e, x=NONE, x8=mat8(0, 16, dtype, 16, ptr=0, scale=0), dx=e, weight=w, rstd=0) == INVALID
        assert norm_grad(grad=e, x=NONE, dx=e, weight=w, rstd=0) == INVALID
        for rows in (0, 3):
            none, none8 = mat(rows, 0, t, ptr=0), mat8(rows, 0, dtype, group, ptr=0, scale=0)
            assert norm_grad(grad=none, x=NONE, x8=none8, dx=none, weight=NONE, rstd=0) == OK
            assert norm_grad(grad=none, x=none, dx=none, weight=NONE, rstd=0) == OK
    assert norm_grad(x=NONE, x8=mat8(3, 16, dtype, group, ptr=0)) == INVALID


@pytest.mark.parametrize("how", (copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))), ids=("copy", "deepcopy", "pickle"))
def test_copies_of_a_rotary(how):
    """A copied model's Rotary reads memory that it holds, not the original's, which may be gone."""
    first = etc.Rotary(64, scaling="linear", factor=4.0, layout="interleaved", scale=0.5)
    freq, r = first.freq, how(first)
    assert r._at == ctypes.addressof(r._desc) and r.freq == freq
    d = etc.RotaryDesc.from_address(r._at)
    assert (list(d.freq[:32]), d.scale, d.pairs, d.layout) == (freq, 0.5, 32, etc.ROTARY_INTERLEAVED)
    if how is not copy.copy:
        assert r._at != first._at
        first._desc.freq[0] = 7.0
        assert r.freq == freq


@pytest.mark.parametrize("kw", (dict(dim=4, factor=1e160), dict(dim=128, base=1e300, factor=1e9)))
def test_a_base_past_64_bits_is_refused(kw):
    with pytest.raises(etc.EtcError, match="infinite"):
        etc.Rotary(scaling="base", **kw)


@pytest.mark.parametrize("kw", (dict(low=-1e308, high=1e308), dict(low=float("-inf"), high=1.0), dict(low=1.0, high=float("inf"))))
def test_a_ramp_past_64_bits_is_refused(kw):
    with pytest.raises(etc.EtcError, match="difference"):
        etc.Rotary(8, scaling="parts", factor=8.0, length=4096.0, **kw)


@pytest.mark.parametrize("dim", ((1 << 32) + 64, (1 << 64) + 2, 64 - (1 << 32), 1 << 31, -2))
def test_a_dim_past_32_bits_is_refused(dim):
    with pytest.raises(ValueError, match="dim"):
        etc.Rotary(dim)
