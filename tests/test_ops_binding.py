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
