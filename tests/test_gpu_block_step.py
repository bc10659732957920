"""The operators around a block's projections together, as a training step uses
them: norm with 8-bit output, product, rotary positions, and the way back
with activations kept in 8 bits, against the same in 64 bits; on other streams, on
streams that have yet to write the inputs, and in graphs."""
import numpy as np
import pytest
import torch

import block_ref
from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


class Step:
    """The input of a block's attention: h = x + residual, n = norm(h) in 8 bits, y = n W^T + b, the first heads of y
    turned.  Backward of sum(c * y) + sum(d * h), with h and n kept in 8 bits."""

    def __init__(self, tokens, hidden, heads, others, head_dim, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        rand = lambda *s, std=1.0: torch.randn(*s, generator=gen, device=DEV) * std  # noqa: E731
        act = lambda n, t=BF16: torch.empty(tokens, n, dtype=t, device=DEV)  # noqa: E731
        bytes8 = lambda r, c: torch.empty(r, c, dtype=torch.int8, device=DEV)  # noqa: E731
        self.tokens, self.hidden, self.heads, self.head_dim = tokens, hidden, heads, head_dim
        n = (heads + others) * head_dim
        self.turned, self.n = heads * head_dim, n
        self.x, self.residual, self.norm_weight = rand(tokens, hidden).bfloat16(), rand(tokens, hidden).bfloat16(), (1 + 0.1 * rand(hidden)).bfloat16()
        self.weight, self.bias = rand(n, hidden, std=hidden ** -0.5).bfloat16(), rand(n, std=0.1).bfloat16()
        self.c, self.d = rand(tokens, n).bfloat16(), rand(tokens, hidden).bfloat16()
        self.positions = torch.arange(tokens, device=DEV) % 1000
        self.rotary = etc.Rotary(head_dim)
        self.w8 = etc.Matrix8(bytes8(n, hidden), torch.empty(n, device=DEV))
        self.wt = etc.Matrix8(bytes8(hidden, n))  # the data transposed, its scales go into the gradient
        self.h, self.y, self.dy, self.dh = act(hidden), act(n), act(n), act(hidden)
        self.n8 = etc.Matrix8(bytes8(tokens, hidden), torch.empty(tokens, device=DEV))
        self.h8 = etc.Matrix8(bytes8(tokens, hidden), torch.empty(tokens, -(-hidden // 128), device=DEV), 128)
        self.g8 = etc.Matrix8(bytes8(tokens, n), torch.empty(tokens, device=DEV))
        self.rstd, self.dnorm = torch.empty(tokens, device=DEV), torch.empty(hidden, device=DEV)
        self.dn, self.n16 = act(hidden), act(hidden)
        self.work = torch.empty(etc.etc_norm_grad_bytes(tokens, hidden), dtype=torch.uint8, device=DEV)
        self.inputs = [self.x, self.residual, self.norm_weight, self.weight, self.bias, self.c, self.d, self.positions]
        self.outputs = [self.h, self.y, self.n8.data, self.n8.scale, self.h8.data, self.h8.scale, self.rstd, self.dn, self.dh,
                        self.dnorm, self.n16, self.w8.data, self.w8.scale]

    def run(self, stream=None):
        s = dict(stream=stream)
        # the weight's 8 bits are made once a step; their transpose is a copy
        etc.etc_store8(self.weight, self.w8, **s)
        etc.etc_norm(self.x, self.norm_weight, out8=self.n8, residual=self.residual, sum=self.h, rstd=self.rstd, eps=1e-5, **s)
        etc.etc_store8(self.h, self.h8, **s)
        etc.etc_matmul8(self.n8, self.w8, self.y, bias=self.bias, **s)
        heads = self.y[:, :self.turned]
        etc.etc_rotary(heads, heads, self.positions, self.rotary, self.head_dim, **s)

    def back(self, stream=None):
        s = dict(stream=stream)
        heads = self.dy[:, :self.turned]
        etc.etc_rotary(heads, heads, self.positions, self.rotary, self.head_dim, backward=True, **s)
        etc.etc_store8(self.dy, self.g8, col_scale=self.w8.scale, **s)
        etc.etc_matmul8(self.g8, self.wt, self.dn, **s)
        etc.etc_load8(self.n8, self.n16, **s)  # for the weight's gradient, dy^T n, a product of the caller's
        etc.etc_norm_grad(self.dn, self.h8, self.norm_weight, self.rstd, self.dh, dsum=self.d, dweight=self.dnorm, workspace=self.work, **s)

    def all(self, stream=None):
        self.run(stream)
        on = torch.cuda.current_stream() if stream is None else stream
        with torch.cuda.stream(on):
            self.wt.data.copy_(self.w8.data.t())
            self.dy.copy_(self.c)
        self.back(stream)


def off(got, want):
    got, want = got.double().cpu(), torch.as_tensor(want, dtype=torch.float64)
    return float((got - want).norm() / want.norm())


SIZES = [(200, 256, 4, 2, 64), (67, 680, 3, 1, 40), (1, 512, 8, 2, 64), (300, 2048, 10, 2, 128)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_a_step_and_its_way_back(size):
    """Against 64 bits without any rounding.  int8 with a scale for `count` normal numbers has steps of a / 127
    with a = their largest, sqrt(2 ln count) standard deviations or so (5 at most here), so an error of a / (127
    sqrt(12)) = 1.1 % of their root mean square; bf16's is 2^-9 / sqrt(3) or so.  y has that of n and of W:
    1.7 % with bf16's.  dn has that of dy and of W, and dh that of dn and of h: 2.0 %; twice that is allowed."""
    say("block step", size)
    s = Step(*size, seed=1)
    s.all()
    torch.cuda.synchronize()
    x, res, nw, w, b, c, d = (t.double().cpu().requires_grad_() for t in
                              (s.x, s.residual, s.norm_weight, s.weight, s.bias, s.c, s.d))
    h = x + res
    n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-5) * nw
    y = n @ w.t() + b
    # the rotation as a product with the real and imaginary part of e^(i angle)
    t, p = size[0], size[4] // 2
    freq = torch.from_numpy(block_ref.frequencies(size[4]))
    angle = s.positions.cpu().double()[:, None] * freq
    heads = y[:, :s.turned].reshape(t, s.heads, 2, p)
    a, e = heads[:, :, 0], heads[:, :, 1]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    turned = torch.stack((a * cos - e * sin, e * cos + a * sin), 2).reshape(t, s.turned)
    y = torch.cat((turned, y[:, s.turned:]), 1)
    ((c * y).sum() + (d * h).sum()).backward()
    assert off(s.h, h.detach()) < 2.0 ** -8
    assert off(s.n16, n.detach()) < 2 * 0.012
    assert off(s.y, y.detach()) < 2 * 0.017
    assert off(s.dh, x.grad) < 2 * 0.02 and torch.equal(x.grad, res.grad)
    assert off(s.dnorm, nw.grad) < 2 * 0.02
    dw = s.dy.float().t() @ s.n16.float()  # the caller's product
    assert off(dw, w.grad) < 2 * 0.017


@pytest.mark.parametrize("given", (True, False), ids=("stream-given", "current-stream"))
@pytest.mark.parametrize("size", SIZES[:2], ids=lambda s: "-".join(map(str, s)))
def test_inputs_that_the_stream_has_yet_to_write(size, given):
    busy = torch.zeros(1 << 28, device=DEV)
    say("block step on a busy stream", size, given)
    s = Step(*size, seed=2)
    s.all()
    torch.cuda.synchronize()
    want, late = [t.clone() for t in s.outputs], [t.clone() for t in s.inputs]
    for t in s.inputs + s.outputs:
        t.zero_()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(60):
            busy.add_(1.0)
        for t, u in zip(s.inputs, late):
            t.copy_(u)
        if not given:
            s.all()
    if given:
        s.all(stream)
    assert not stream.query(), "the stream was idle before the call: nothing was shown"
    stream.synchronize()
    assert all(torch.equal(t, u) for t, u in zip(s.outputs, want))


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_in_graphs(size):
    """A step captured and replayed, two graphs that share all buffers in turn, with eager steps between them."""
    say("block step in graphs", size)
    s = Step(*size, seed=3)
    s.all()
    torch.cuda.synchronize()
    want = [t.clone() for t in s.outputs]
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.all()
        graphs.append(g)
    for replay in range(4):
        for t in s.outputs:
            t.zero_()
        torch.cuda.synchronize()
        graphs[replay % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, u) for t, u in zip(s.outputs, want)), replay
        for t in s.outputs:
            t.zero_()
        s.all()
        torch.cuda.synchronize()
        assert all(torch.equal(t, u) for t, u in zip(s.outputs, want)), replay


def test_refusals_on_the_gpu():
    """Tensors of other places are refused before anything runs."""
    say("block refusals")
    x, w, q = torch.zeros(4, 64, dtype=BF16, device=DEV), torch.zeros(64, dtype=BF16, device=DEV), torch.zeros(4, 64, dtype=torch.int8, device=DEV)
    s, m, pos = torch.zeros(4, device=DEV), None, torch.zeros(4, dtype=torch.int64, device=DEV)
    m = etc.Matrix8(q, s)
    wrong = [
        lambda: etc.etc_norm(x, w.cpu(), out=x), lambda: etc.etc_norm(x.cpu(), w, out=x), lambda: etc.etc_norm(x, w, out=x, rstd=s.cpu()),
        lambda: etc.etc_norm(x, w, out8=etc.Matrix8(q.cpu(), s)), lambda: etc.etc_norm(x, w, out8=etc.Matrix8(q, s.cpu())),
        lambda: etc.etc_norm_grad(x, x, w, s.cpu(), x), lambda: etc.etc_store8(x, m, col_scale=w.float().cpu()),
        lambda: etc.etc_load8(m, x.cpu()), lambda: etc.etc_matmul8(m, etc.Matrix8(q.cpu(), s), x[:, :4]),
        lambda: etc.etc_rotary(x, x, pos.cpu(), etc.Rotary(64), 64), lambda: etc.etc_rotary(x, x.cpu(), pos, etc.Rotary(64), 64),
    ]
    for k, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            say("not refused:", k)
    refused = [
        lambda: etc.etc_norm(x, w, out=x, sum=x), lambda: etc.etc_norm(x, w, out=x, eps=0.0),
        lambda: etc.etc_norm_grad(x, x, w, s, x, dweight=torch.zeros(64, device=DEV)),
        lambda: etc.etc_matmul8(m, m, x), lambda: etc.etc_rotary(x, x, pos, etc.Rotary(128), 64),
        lambda: etc.etc_matmul8(m, etc.Matrix8(q.view(torch.float8_e4m3fn), s), x[:, :4]), lambda: etc.etc_load8(etc.Matrix8(q), x),
        lambda: etc.etc_rotary(x, x[:1].expand(4, 64), pos, etc.Rotary(64), 64),
    ]
    for k, call in enumerate(refused):
        with pytest.raises(etc.EtcError):
            call()
            say("not refused:", k)
    torch.cuda.synchronize()
    assert not bool(x.any()) and not bool(q.any()) and not bool(s.any())
