"""The operators around a block's projections on the GPU at the ends of what they
take."""
import pytest
import torch

from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DT8 = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kept", (None, "i8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_backward_of_no_tokens(kept, dtype):
    """A rank without tokens in a micro-batch: the weight's gradient is 0, or what it was."""
    say("norm_grad of no tokens", kept, dtype)
    e, rstd = torch.empty(0, 300, dtype=dtype, device=DEV), torch.empty(0, device=DEV)
    for group in (0, 32):
        x = e if kept is None else etc.Matrix8(torch.empty(0, 300, dtype=DT8[kept], device=DEV),
                                               torch.empty(0, 10 if group else 1, device=DEV), group)
        for accumulate in (False, True):
            dw = torch.full((300,), 3.0, device=DEV)
            etc.etc_norm_grad(e, x, torch.ones(300, dtype=dtype, device=DEV), rstd, torch.empty_like(e), dweight=dw, accumulate=accumulate)
            assert bool((dw == (3.0 if accumulate else 0.0)).all())
        etc.etc_norm_grad(e, x, torch.ones(300, dtype=dtype, device=DEV), rstd, torch.empty_like(e))


@pytest.mark.parametrize("rows,cols,dtype", ((1, 4096, "bf16"), (5, 9, "f32"), (64, 4096, "bf16"), (256, 681, "bf16"), (1021, 681, "f32"),
                                             (1024, 2048, "bf16"), (600, 129, "bf16"), (128, 16384, "bf16"), (100, 8191, "f32"),
                                             (1025, 681, "bf16"), (5000, 256, "bf16")))
def test_order_of_the_weight_gradients_sums(rows, cols, dtype):
    """It depends on the sizes and on whether dx is grad or x itself, and on nothing else: not on which of the two, on dsum, nor on
    what the workspace held."""
    say("weight gradient, in place and not", rows, cols, dtype)
    gen = torch.Generator(device=DEV).manual_seed(rows)
    grad, x, dsum = (torch.randn(rows, cols, device=DEV, generator=gen).to(DT[dtype]) for _ in range(3))
    weight = torch.randn(cols, device=DEV, generator=gen).to(DT[dtype])
    rstd, before = torch.rand(rows, device=DEV, generator=gen) + 0.5, torch.randn(cols, device=DEV, generator=gen)
    ws = torch.empty(etc.etc_norm_grad_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    for accumulate in (False, True):
        first = {}
        for to in ("apart", "grad", "x", "dsum"):
            g, h, d, dw = grad.clone(), x.clone(), dsum.clone(), before.clone()
            dx = {"apart": torch.empty_like(g), "grad": g, "x": h, "dsum": d}[to]
            ws.random_(0, 256)
            etc.etc_norm_grad(g, h, weight, rstd, dx, dsum=d, dweight=dw, workspace=ws, accumulate=accumulate)
            then = first.setdefault(to in ("grad", "x"), dw)
            assert torch.equal(dw, then), (to, accumulate)
            for name, now, then in (("grad", g, grad), ("x", h, x), ("dsum", d, dsum)):
                assert name == to or torch.equal(now, then), (to, name)
