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


@pytest.mark.parametrize("m,n", (((1 << 19) + 5, 9), (3, (1 << 20) + 3)))
def test_products_of_several_launches(m, n):
    """More rows, or columns, than a launch takes: the next one's operands, scales and bias follow on.  Whole numbers and powers
    of two: exact."""
    say("matmul8 in several launches", m, n)
    gen = torch.Generator(device=DEV).manual_seed(m)
    x, w = (torch.randint(-127, 128, (r, 33), generator=gen, device=DEV, dtype=torch.int8) for r in (m, n))
    sx, sw = (torch.exp2(torch.randint(-2, 3, (r,), generator=gen, device=DEV).float()) for r in (m, n))
    bias = torch.randint(-9, 10, (n,), generator=gen, device=DEV).float()
    out = torch.full((m + 1, n), 7.0, device=DEV)
    etc.etc_matmul8(etc.Matrix8(x, sx), etc.Matrix8(w, sw), out[:m], bias=bias)
    want = (x.double() @ w.double().t().contiguous()) * sx.double()[:, None] * sw.double() + bias.double()
    assert torch.equal(out[:m].double(), want) and bool((out[m] == 7).all())


def test_norms_of_several_launches():
    """Rows past the 2^32 lanes of a launch.  A row's elements are 2^e or -2^e, so its rms is 2^e, and every result is exact."""
    rows = (1 << 26) + 3
    say("norm in several launches", rows)
    gen = torch.Generator(device=DEV).manual_seed(5)
    sign = torch.randint(0, 2, (rows, 8), generator=gen, device=DEV, dtype=torch.int8) * 2 - 1
    e = torch.arange(rows, device=DEV) % 5
    x = (sign * torch.exp2(e.float()).to(torch.bfloat16)[:, None])
    w, r = torch.ones(8, dtype=torch.bfloat16, device=DEV), torch.empty(rows, device=DEV)
    m8, out = etc.Matrix8(torch.empty_like(sign), torch.empty(rows, device=DEV)), torch.empty_like(x)
    etc.etc_norm(x, w, out=out, out8=m8, rstd=r, eps=2.0 ** -40)
    assert torch.equal(r, torch.exp2(-e.float())) and torch.equal(out, sign.to(torch.bfloat16))
    assert torch.equal(m8.data, sign * 127) and bool((m8.scale == torch.tensor(1.0, device=DEV) / 127).all())
    etc.etc_store8(x, m8)
    assert torch.equal(m8.data, sign * 127) and torch.equal(m8.scale, torch.exp2(e.float()) / 127)
    del m8
    grad = torch.randint(-3, 4, (rows, 8), generator=gen, device=DEV, dtype=torch.int8).to(torch.bfloat16)
    etc.etc_norm_grad(grad, x, w, r, out)
    for at in range(0, rows, 1 << 24):
        part = slice(at, min(rows, at + (1 << 24)))
        g, n = grad[part].float(), sign[part].float()
        want = (g - n * (g * n).mean(1, keepdim=True)) * r[part, None]
        assert torch.equal(out[part].float(), want), at
