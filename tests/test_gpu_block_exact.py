"""The norm's weight gradient where it has one right answer (block_exact.py):
equality, on every path that its rows and columns lead to, wherever dx goes."""
import numpy as np
import pytest
import torch

import block_exact
import block_ref
from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def on_gpu(x, dtype):
    return torch.from_numpy(x).to(DEV).to(dtype)


def kept8(x, scale, kept, group):
    """x (whole numbers of -3 .. 3) and scales as a Matrix8."""
    if kept == "i8":
        return etc.Matrix8(torch.from_numpy(x).to(DEV), torch.from_numpy(scale).to(DEV), group)
    codes = np.zeros(7, np.uint8)
    for v in range(-3, 4):
        codes[v + 3] = np.flatnonzero(block_ref.E4M3 == v)[0]
    return etc.Matrix8(torch.from_numpy(codes[x + 3]).to(DEV).view(torch.float8_e4m3fn), torch.from_numpy(scale).to(DEV), group)


@pytest.mark.parametrize("case", block_exact.DWEIGHT, ids=str)
def test_weight_gradient(case):
    say("exact weight gradient", case)
    rows, cols, dtype, kept, group = case
    grad, x, scale, r, before = block_exact.dweight_case(case)
    sums = block_exact.dweight_sums(grad, x, scale, group, r)
    weight, rstd = torch.ones(cols, dtype=DT[dtype], device=DEV), on_gpu(r, torch.float32)
    ws = torch.empty(etc.etc_norm_grad_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    for accumulate, want in ((False, sums), (True, sums + before)):
        for to in ("apart", "grad", "x", "dsum"):
            g, dw = on_gpu(grad, DT[dtype]), on_gpu(before, torch.float32)
            source = kept8(x, scale, kept, group) if kept else on_gpu(x, DT[dtype])
            dsum = torch.ones_like(g) if to == "dsum" else None
            if to == "x" and kept:
                continue
            dx = {"apart": torch.empty_like(g), "grad": g, "x": source, "dsum": dsum}[to]
            etc.etc_norm_grad(g, source, weight, rstd, dx, dsum=dsum, dweight=dw, workspace=ws, accumulate=accumulate)
            got = dw.cpu().numpy()
            bad = got != want
            assert not bad.any(), (case, accumulate, to, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3])
