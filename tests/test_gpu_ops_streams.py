"""Each operator works on the stream it is given, or the current one: called
while that stream is still busy with what comes before the operator's inputs, it
sees the inputs all the same."""
import pytest
import torch

from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rand(gen, *shape, dtype=BF16):
    return torch.randn(*shape, generator=gen, device=DEV).to(dtype)


def operators(tokens):
    """{name: (inputs, outputs, call(stream))} on `tokens` rows; outputs that are also inputs are among the inputs."""
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    rows, cols, drop = 50, 136, etc.Dropout(0.1, 21)
    ids = torch.randint(-2, rows + 2, (tokens,), generator=gen, device=DEV)
    table, x, bias, grad = rand(gen, rows, cols), rand(gen, tokens, cols), rand(gen, cols), rand(gen, tokens, cols)
    out, dx = (torch.empty(tokens, cols, dtype=BF16, device=DEV) for _ in range(2))
    dtable, dbias = torch.empty(rows, cols, device=DEV), torch.empty(cols, device=DEV)
    ws = torch.empty(max(etc.etc_embed_grad_bytes(tokens, rows, cols), etc.etc_dropout_grad_bytes(tokens, cols)),
                     dtype=torch.uint8, device=DEV)
    arenas = [rand(gen, rows * cols)] + [rand(gen, rows * cols, dtype=F32).abs_() for _ in range(3)]
    grads, clip = rand(gen, rows * cols, dtype=F32), torch.full((1,), 0.25, device=DEV)
    return {
        "embed": ([ids, table], [out], lambda s: etc.etc_embed(ids, table, out, scale=2.0, dropout=drop, stream=s)),
        "embed_grad": ([ids, grad], [dtable], lambda s: etc.etc_embed_grad(ids, grad, dtable, ws, dropout=drop, stream=s)),
        "dropout": ([x, bias, grad], [out], lambda s: etc.etc_dropout(x, out, drop, bias=bias, residual=grad, stream=s)),
        "dropout_grad": ([grad], [dx, dbias],
                         lambda s: etc.etc_dropout_grad(grad, dx, drop, dbias=dbias, workspace=ws, stream=s)),
        "dropout_dx": ([grad], [dx], lambda s: etc.etc_dropout_grad(grad, dx, drop, stream=s)),
        "adam": (arenas + [grads, clip], arenas,
                 lambda s: etc.etc_adam(arenas, grads, step=3, lr=1e-2, grad_scale=clip, stream=s)),
    }


@pytest.mark.parametrize("given", (True, False), ids=("stream-given", "current-stream"))
@pytest.mark.parametrize("tokens", (300, 3000))
def test_inputs_that_the_stream_has_yet_to_write(tokens, given):
    busy = torch.zeros(1 << 28, device=DEV)  # 1 GB: a third of a millisecond a pass
    s = torch.cuda.Stream()
    for name, (inputs, outputs, call) in operators(tokens).items():
        say("streams", name, tokens, given)
        late = [x.clone() for x in inputs]
        call(None)
        torch.cuda.synchronize()
        want = [x.clone() for x in outputs]
        for x in inputs + outputs:
            x.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(60):
                busy.add_(1.0)
            for x in outputs:
                x.fill_(7.0)
            for x, y in zip(inputs, late):
                x.copy_(y)
            if not given:
                call(None)
        if given:
            call(s)
        assert not s.query(), "the stream was idle before the call: nothing was shown"
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outputs, want)), name
        torch.cuda.synchronize()
