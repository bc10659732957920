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
