"""A table's gradient does not depend on how many ranks share the table: the
shares' rows, each rank's computed from the same tokens and gradients, are the
whole table's, bit for bit, however long the batch is."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

CASES = [
    # tokens, cols, vocabulary, dtype, p, kind of ids
    (300, 200, 96, "bf16", 0.1, "log"),
    (700, 520, 96, "bf16", 0.1, "log"),
    (129, 8192, 64, "bf16", 0.0, "log"),
    (65, 8192, 64, "f32", 0.1, "log"),
    (1500, 333, 1000, "f32", 0.0, "log"),
    (2049, 256, 48, "bf16", 0.1, "even"),
    (8192, 512, 4000, "bf16", 0.0, "log"),
    (16384, 2048, 5024, "bf16", 0.1, "log"),
    (16411, 17, 480, "f32", 0.25, "log"),
    (40000, 100, 16, "bf16", 0.0, "even"),
    (70001, 24, 50304, "f32", 0.1, "log"),
]


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_shares_are_the_whole_table(case, accumulate):
    tokens, cols, vocab, dtype, p, kind = case
    say("shares of a table's gradient", case, accumulate)
    rng = np.random.default_rng([tokens, cols, vocab])
    v = (np.exp(rng.random(tokens) * np.log(vocab + 1)) - 1).astype(np.int64) if kind == "log" else rng.integers(0, vocab, tokens)
    v[::13] = -1
    v[7::101] = vocab + 3
    ids = torch.from_numpy(v).to(DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    grad = torch.randn(tokens, cols, generator=gen, device=DEV).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    before = torch.randn(vocab, cols, generator=gen, device=DEV)
    ws = torch.empty(etc.etc_embed_grad_bytes(tokens, vocab, cols), dtype=torch.uint8, device=DEV)
    drop = etc.Dropout(p, 77, row0=5)

    def gradient(row0, rows):
        d = before[row0:row0 + rows].clone()
        etc.etc_embed_grad(ids, grad, d, ws, row0=row0, scale=1.25, dropout=drop, accumulate=accumulate)
        return d

    whole = gradient(0, vocab)
    for tp in (2, 4, 8):
        n = vocab // tp
        assert torch.equal(torch.cat([gradient(r * n, n) for r in range(tp)]), whole), tp
    # a share of any place and size
    assert torch.equal(gradient(3, vocab - 7), whole[3:vocab - 4])
    assert torch.equal(gradient(vocab // 3, 1), whole[vocab // 3:vocab // 3 + 1])
