"""The operators around a block's projections on the GPU at the ends of what they
take: batches without tokens, and sizes past what one launch has."""
import pytest
import torch

from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

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
