"""etc_norm's 8 bits against its definition bit for bit, and with an eps so small
that 1 / sqrt(eps) times the factor of a row of zeros is past 32 bits."""
import numpy as np
import pytest
import torch

import block_ref
from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

DT8 = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
COLS = (3, 40, 250, 1000, 33000)  # rows of less than a block, of few lanes, of a wavefront, of a workgroup, and longer


def matrix8(rows, cols, eight):
    return etc.Matrix8(torch.full((rows, cols), 0x5A, dtype=torch.uint8, device=DEV).view(DT8[eight]),
                       torch.empty(rows, device=DEV))


def whole(rng, rows, cols):
    """-3 .. 3 without 0."""
    return (rng.integers(1, 4, (rows, cols)) * rng.choice((-1, 1), (rows, cols))).astype(np.float32)


@pytest.mark.parametrize("eight", ("i8", "e4m3"))
@pytest.mark.parametrize("eps", (1e-6, 1e-12, 1e-13, 1e-30, 2.0 ** -126))
@pytest.mark.parametrize("cols", COLS)
def test_small_rows_with_a_small_eps(cols, eps, eight):
    """Zeros stay zeros, and rows far below 1 are what they should be.  Elements are whole numbers times a power of two and
    weights powers of two, so s * weight is exact; squares vanish beside eps or are of its order or above, and normal."""
    say("norm in 8 bits, small eps", cols, eps, eight)
    rng = np.random.default_rng([cols, len(eight)])
    x = whole(rng, 9, cols) * np.exp2([[0.0], [-10], [-40], [-52], [-80], [-100], [-110], [-122], [-124]]).astype(np.float32)
    x[0] = 0.0
    x[2, 1:] = 0.0  # a single element
    x[5, 0] = -0.0
    w = np.exp2(rng.integers(-1, 2, cols)).astype(np.float32)
    want = block_ref.norm(x, w, None, eps)
    for dtype in (torch.float32, torch.bfloat16):  # which holds x and w too
        for with_out in (False, True):
            out = torch.empty(9, cols, dtype=dtype, device=DEV) if with_out else None
            m8, back = matrix8(9, cols, eight), torch.empty(9, cols, device=DEV)
            etc.etc_norm(torch.from_numpy(x).to(DEV).to(dtype), torch.from_numpy(w).to(DEV).to(dtype), out=out, out8=m8, eps=eps)
            etc.etc_load8(m8, back)
            data, scale = m8.data.view(torch.uint8).cpu().numpy(), m8.scale.cpu().numpy()
            assert not back[0].any() and not block_ref.values8(data[:1], eight).any()
            assert scale[0] == block_ref.LEAST / np.float32(block_ref.TOP[eight])
            assert bool(back.isfinite().all())
            block_ref.check_norm8(data, scale.astype(np.float64), eight, want["out"])
            if with_out:
                assert not out[0].any() and bool(out.isfinite().all())


@pytest.mark.parametrize("eight", ("i8", "e4m3"))
@pytest.mark.parametrize("cols", COLS)
def test_the_8_bits_of_the_norm_are_those_of_its_output(cols, eight):
    """out8 is out, where that is in 32 bits, through the definition's steps: the same scales, the same data."""
    say("norm in 8 bits, bit for bit", cols, eight)
    rng = np.random.default_rng([cols, 1 + len(eight)])
    x, res, w = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV) for s in ((70, cols), (70, cols), (cols,)))
    out, m8, alone = torch.empty(70, cols, device=DEV), matrix8(70, cols, eight), matrix8(70, cols, eight)
    etc.etc_norm(x, w, out=out, out8=m8, residual=res, eps=1e-5)
    etc.etc_norm(x, w, out8=alone, residual=res, eps=1e-5)
    data, scale = block_ref.store8(out.cpu().numpy(), eight, 0)
    for got in (m8, alone):
        assert np.array_equal(got.scale.cpu().numpy(), scale[:, 0])
        assert np.array_equal(got.data.view(torch.uint8).cpu().numpy(), data)
    stored = matrix8(70, cols, eight)
    etc.etc_store8(out, stored)
    assert torch.equal(stored.data.view(torch.uint8), m8.data.view(torch.uint8)) and torch.equal(stored.scale, m8.scale)
