"""The README's lines around a projection, run as they stand, against the plain
implementations in 64 bits."""
import os

import numpy as np
import pytest
import torch

import block_ref
from gpu_util import DEV, say
from paper_2607_04749_amd import etc
from test_gpu_ops import close, rand, workspace

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def snippet():
    blocks = [b.split("```")[0] for b in open(README).read().split("```python\n")[1:]]
    found = [b for b in blocks if "etc.etc_matmul8(" in b]
    assert len(found) == 1
    return found[0]


@pytest.mark.parametrize("tokens,hidden,heads,others,head_dim", ((200, 256, 5, 2, 64), (1, 520, 3, 1, 40)))
def test_readme_around_a_projection(tokens, hidden, heads, others, head_dim):
    say("README around a projection", tokens, hidden)
    rng = np.random.default_rng(tokens)
    columns, turned = (heads + others) * head_dim, heads * head_dim
    x, xn, _ = rand(rng, tokens, hidden, "bf16")
    h, hn, _ = rand(rng, tokens, hidden, "bf16")
    w, wn, _ = rand(rng, 1, hidden, "bf16")
    dqkv, gn, _ = rand(rng, tokens, columns, "bf16")
    dy, dyn, _ = rand(rng, tokens, hidden, "bf16")
    dh, dhn, _ = rand(rng, tokens, hidden, "bf16")
    dw, before, _ = rand(rng, 1, hidden, "f32")
    wd = rng.integers(-127, 128, (columns, hidden), dtype=np.int64).astype(np.int8)
    ws = rng.random(columns).astype(np.float32)
    w8 = etc.Matrix8(torch.from_numpy(wd).to(DEV), torch.from_numpy(ws).to(DEV))
    qkv = torch.empty(tokens, columns, dtype=torch.bfloat16, device=DEV)
    pos = rng.integers(0, 4096, tokens)
    names = dict(etc=etc, torch=torch, tokens=tokens, hidden=hidden, head_dim=head_dim, x=x, h=h, norm_weight=w[0], w8=w8, qkv=qkv,
                 qk=qkv[:, :turned], dqk=dqkv[:, :turned], positions=torch.from_numpy(pos).to(DEV), rstd=torch.empty(tokens, device=DEV),
                 dy=dy, dh=dh, dw=dw[0], work=workspace(etc.etc_norm_grad_bytes(tokens, hidden))[0])
    exec(snippet(), names)
    torch.cuda.synchronize()
    q8, kept, freq = names["q8"], names["kept"], np.array(names["rotary"].freq)
    norm = block_ref.norm(xn, wn[0], hn, 1e-6)  # etc_norm's own eps
    close(h, norm["sum"], "h")
    close(names["rstd"], norm["rstd"], "rstd")
    data, scale = q8.data.cpu().numpy(), q8.scale.cpu().numpy()
    block_ref.check_norm8(data.view(np.uint8), scale.astype(np.float64), "i8", norm["out"])
    plain = torch.empty_like(qkv)
    etc.etc_matmul8(q8, w8, plain)
    close(plain, block_ref.matmul8(data, wd, scale, ws), "qkv")
    close(qkv[:, :turned], block_ref.rotary(plain[:, :turned].float().cpu().numpy(), pos, freq, head_dim), "qk")
    assert torch.equal(qkv[:, turned:], plain[:, turned:])
    bytes8, scales = block_ref.store8(h.float().cpu().numpy(), "i8", 128)
    assert np.array_equal(kept.data.cpu().numpy().view(np.uint8), bytes8) and np.array_equal(kept.scale.cpu().numpy(), scales)
    close(names["dqk"], block_ref.rotary(gn[:, :turned], pos, freq, head_dim, backward=True), "dqk")
    assert np.array_equal(dqkv[:, turned:].float().cpu().numpy(), gn[:, turned:])
    back = block_ref.norm_grad(dyn, block_ref.load8(bytes8, scales, "i8", 128), wn[0], names["rstd"].cpu().numpy(), dhn, before[0], True, True)
    close(dh, back["dx"], "dh")
    close(dw[0], back["dweight"], "dw")
