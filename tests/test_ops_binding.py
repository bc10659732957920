"""What the binding of the operators hands to the library, without a GPU: host
tensors stand for device tensors, and the library's calls are recorded."""
import pytest
import torch

from paper_2607_04749_amd import etc

BF16, F32 = torch.bfloat16, torch.float32


class Recorder:
    """Keeps each call's packed arguments, and succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda packed, stream: self.calls.append((name, packed)) or etc.OK


@pytest.fixture
def calls(monkeypatch):
    library = Recorder()
    monkeypatch.setattr(etc, "_lib", library)
    monkeypatch.setattr(etc, "_device_of", lambda x, what: x.get_device())
    return library.calls


def test_rows_of_no_columns_are_counted(calls):
    """Tokens of any shape: [4, 6] into [4, 6, 0] are 24 rows, as in [24, 0]."""
    tokens, table = torch.zeros(4, 6, dtype=torch.int64), torch.zeros(9, 0, dtype=BF16)
    etc.etc_embed(tokens, table, torch.zeros(4, 6, 0, dtype=BF16), stream=0)
    etc.etc_embed(tokens, table, torch.zeros(24, 0, dtype=BF16), stream=0)
    out = [etc._EMBED.unpack(packed)[20:26] for _, packed in calls]
    assert [m[1:3] for m in out] == [(24, 0), (24, 0)]


def test_an_empty_tensor_is_not_an_absent_one(calls):
    """None stands for a bias, residual or bias gradient that is not wanted; an
    empty tensor, whose address is 0 as well, has the wrong size and is refused."""
    x, drop = torch.zeros(3, 16, dtype=BF16), etc.Dropout(0.1, 1)
    for empty in (x[:0], x[:, :0], x[0, :0], torch.zeros(0, dtype=BF16)):
        for name in ("bias", "residual"):
            with pytest.raises(ValueError, match=name):
                etc.etc_dropout(x, x, drop, stream=0, **{name: empty})
        with pytest.raises(ValueError, match="dbias"):
            etc.etc_dropout_grad(x, x, drop, dbias=empty.float(), stream=0)
    with pytest.raises(ValueError, match="dbias"):  # no rows, but columns whose sums are zeros
        etc.etc_dropout_grad(x[:0], x[:0], drop, dbias=x[0, :0].float(), stream=0)
    assert not calls
    # where x is empty too they are of its size
    etc.etc_dropout(x[:0], x[:0], drop, bias=x[0], residual=x[:0], stream=0)
    etc.etc_dropout(x[:, :0], x[:, :0], drop, bias=x[0, :0], residual=x[:, :0], stream=0)
    etc.etc_dropout_grad(x[:, :0], x[:, :0], drop, dbias=x[0, :0].float(), stream=0)
    assert len(calls) == 3


def test_adam_takes_no_other_types(calls, monkeypatch):
    """The parameter's arena is bfloat16, the others and the gradients float32,
    each also as bytes; a tensor of another type and enough bytes is refused, and so
    is one of another device."""
    monkeypatch.setattr(etc, "_current_device", lambda: -1)
    n = 64
    right = [torch.zeros(n, dtype=t) for t in (BF16, F32, F32, F32, F32)]

    def step(*tensors):
        etc.etc_adam(tensors[:4], tensors[4], step=1, lr=1e-3, count=n, stream=0)

    for k, wrong in ((0, (F32, torch.float16, torch.int16, torch.int64)),
                     *((k, (BF16, torch.float64, torch.int32, torch.float16)) for k in (1, 2, 3, 4))):
        for dtype in wrong:
            with pytest.raises(ValueError, match="bfloat16" if k == 0 else "float32"):
                step(*right[:k], torch.zeros(2 * n, dtype=dtype), *right[k + 1:])
    for k in range(5):
        with pytest.raises(ValueError, match="bytes"):
            step(*right[:k], right[k][:-1], *right[k + 1:])
        with pytest.raises(ValueError, match="contiguous"):
            step(*right[:k], torch.zeros(2 * n, dtype=right[k].dtype)[::2], *right[k + 1:])
    with monkeypatch.context() as m, pytest.raises(ValueError, match="current GPU"):
        m.setattr(etc, "_current_device", lambda: 1)
        step(*right)
    assert not calls
    step(*right)
    step(*(x.view(torch.uint8) for x in right))
    etc.etc_adam([x.data_ptr() for x in right[:4]], right[4].data_ptr(), step=1, lr=1e-3, count=n, stream=0)
    assert len(calls) == 3 and len({packed for _, packed in calls}) == 1
