"""The operators' sums where they have one right answer (op_exact.py): equality,
at long runs of one id, deep merges, and many rows."""
import numpy as np
import pytest
import torch

import op_exact
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


@pytest.mark.parametrize("case", op_exact.GRAD, ids=str)
def test_table_gradient(case):
    say("exact table gradient", case)
    v, g, before, drop = op_exact.grad_case(case)
    written, added = op_exact.grad_sums(v, g, before, drop)
    ids, grad = torch.from_numpy(v).to(DEV), on_gpu(g, DT[case[5]])
    ws = torch.empty(etc.etc_embed_grad_bytes(g.shape[0], *before.shape), dtype=torch.uint8, device=DEV)
    for accumulate, want in ((False, written), (True, added)):
        dt = on_gpu(before, torch.float32)
        etc.etc_embed_grad(ids, grad, dt, ws, scale=4.0, dropout=etc.Dropout(*drop), accumulate=accumulate)
        got = dt.cpu().numpy()
        bad = got != want
        assert not bad.any(), (case, accumulate, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("case", op_exact.BIAS, ids=str)
def test_bias_gradient(case):
    say("exact bias gradient", case)
    g, before, drop = op_exact.bias_case(case)
    dropped, written, added = op_exact.bias_sums(g, before, drop)
    grad = on_gpu(g, DT[case[3]])
    dx = torch.empty_like(grad)
    ws = torch.empty(etc.etc_dropout_grad_bytes(*g.shape), dtype=torch.uint8, device=DEV)
    for accumulate, want in ((False, written), (True, added)):
        db = on_gpu(before, torch.float32)
        etc.etc_dropout_grad(grad, dx, etc.Dropout(*drop), dbias=db, workspace=ws, accumulate=accumulate)
        assert np.array_equal(db.cpu().numpy(), want), (case, accumulate)
        assert np.array_equal(dx.float().cpu().numpy(), dropped), case
