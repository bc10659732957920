"""The README's lines that use the operators, run as they stand: on each rank of
a tensor-parallel group they give what one rank with the whole vocabulary has."""
import os
import threading

import pytest
import torch

from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
TOKENS, VOCAB, COLS, POSITIONS = 200, 48, 72, 64


def snippet():
    blocks = open(README).read().split("```python\n")[1:]
    found = [b.split("```")[0] for b in blocks if "etc.etc_embed(" in b.split("```")[0]]
    assert len(found) == 1
    return found[0]


class Group:
    """All-reduce among threads, each a rank: the sum of the tensors in the order of the ranks."""

    def __init__(self, size):
        self.given, self.barrier = [None] * size, threading.Barrier(size, timeout=60)

    def of(self, rank):
        def all_reduce(x, group=None):
            self.given[rank] = x
            self.barrier.wait()
            total = torch.stack(self.given).sum(0)
            self.barrier.wait()
            x.copy_(total)
            self.barrier.wait()
        return type("dist", (), {"all_reduce": staticmethod(all_reduce)})


def run(tp, table, names):
    """The README's lines on `tp` ranks: each one's names afterwards."""
    group, ranks, errors, n = Group(tp), [], [], VOCAB // tp
    for r in range(tp):
        mine = dict(names, etc=etc, torch=torch, dist=group.of(r), tp_group=None, table=table[r * n:(r + 1) * n],
                    first_id_of_this_rank=r * n, first_row_of_this_rank=0,
                    share=torch.empty(TOKENS, COLS, dtype=table.dtype, device=DEV),
                    out=torch.empty(TOKENS, COLS, dtype=torch.bfloat16, device=DEV), dtable=torch.zeros(n, COLS, device=DEV))
        w = mine["table"].float().flatten()
        mine["arenas"] = [w.to(torch.bfloat16), w.clone(), torch.zeros_like(w), torch.zeros_like(w)]
        mine["grad_arena"] = mine["dtable"].view(-1)
        ranks.append(mine)

    def rank(mine):
        try:
            exec(snippet(), mine)
        except Exception as e:
            group.barrier.abort()
            errors.append(e)

    threads = [threading.Thread(target=rank, args=(mine,)) for mine in ranks]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    return ranks


def test_readme_on_ranks_of_a_group():
    gen = torch.Generator(device=DEV).manual_seed(3)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    table = normal(VOCAB, COLS).to(torch.bfloat16)
    names = dict(tokens=torch.randint(0, VOCAB, (TOKENS,), generator=gen, device=DEV), rows=torch.arange(TOKENS, device=DEV),
                 pos=torch.arange(TOKENS, device=DEV) % POSITIONS, pos_table=normal(POSITIONS, COLS).to(torch.bfloat16),
                 grad=normal(TOKENS, COLS).to(torch.bfloat16), scale=3.3, step=1, calls_per_step=2, t=1,
                 clip=torch.full((1,), 0.5, device=DEV))
    # one rank with the whole vocabulary, as the README says
    want = torch.empty(TOKENS, COLS, dtype=torch.bfloat16, device=DEV)
    etc.etc_embed(names["tokens"], table, want, scale=names["scale"], positions=names["pos"], pos_table=names["pos_table"],
                  dropout=etc.Dropout(0.1, seed=7, call=2))
    whole = run(1, table, names)[0]
    for tp in (1, 2, 4):
        say("README on", tp, "ranks")
        ranks = run(tp, table, names)
        for mine in ranks:
            assert torch.equal(mine["out"], want), tp
        assert torch.equal(torch.cat([mine["dtable"] for mine in ranks]), whole["dtable"])
        for k in range(4):
            assert torch.equal(torch.cat([mine["arenas"][k] for mine in ranks]), whole["arenas"][k])
