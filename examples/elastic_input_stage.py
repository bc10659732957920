"""A small training job that changes its configuration between two steps and
goes on as if nothing had happened, bit for bit.

The input stage of a GPT (this repository's tiny one): token and position
embedding with dropout, and a block's epilogue (bias, dropout, residual) behind
it, trained towards random targets.  The tables and the bias live in the four
state arenas of their tensor-parallel ranks, where etc_plan lays them out; all
ranks of a configuration run on one GPU here, one after another.

  step       etc_embed on every rank's share of the vocabulary, the shares' sum
             with scale, positions and dropout (etc_embed again), the epilogue
             (etc_dropout), the way back (etc_dropout_grad, etc_embed_grad) and
             the optimizer (etc_adam) over every rank's arenas
  reshard    etc_pack on the old ranks, etc_unpack on the new ones

A dropped element depends on (seed, call, row, column), a table's row sums its
tokens in an order that the batch's ids alone decide, and Adam treats each element
alone, so what a step computes does not depend on how many ranks share the
tables: six steps with a change from TP 2 to TP 4 after the third end in the
states of six steps on TP 2.

  python examples/elastic_input_stage.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_04749_amd import etc  # noqa: E402
from paper_2607_04749_amd.workloads import TINY_GPT, Parallel  # noqa: E402

DEV = "cuda"
MODEL, OLD, NEW = TINY_GPT, Parallel(2, 1), Parallel(4, 1)
SEQUENCES, LENGTH = 4, 128
P, SCALE, LR = 0.1, MODEL.hidden ** 0.5, 1e-3
DTYPES = (torch.bfloat16, torch.float32, torch.float32, torch.float32)


class Rank:
    """A rank's arenas, gradient arena, and its pieces of the tensors by name."""

    def __init__(self, plan, side, rank):
        n = plan.arena_elems(side, rank)
        self.arenas = [torch.zeros(n, dtype=t, device=DEV) for t in DTYPES]
        self.grads = torch.zeros(n, device=DEV)
        self.pieces = {p["name"]: p for p in plan.pieces(side, rank)}

    def view(self, name, flat):
        p = self.pieces[name]
        rows, cols = p["r1"] - p["r0"], p["c1"] - p["c0"]
        return flat[p["off"]:p["off"] + rows * cols].view(rows, cols)

    def param(self, name):
        return self.view(name, self.arenas[0])

    def grad(self, name):
        return self.view(name, self.grads)


def fresh_ranks(plan, side, world, seed=None):
    """The ranks of one side; with a seed, their shares of random tensors."""
    ranks = [Rank(plan, side, r) for r in range(world)]
    for rank in ranks if seed is not None else ():
        for name, p in rank.pieces.items():
            gen = torch.Generator(device=DEV).manual_seed(seed + p["tensor"])
            full = torch.randn(p["full_rows"], p["full_cols"], generator=gen, device=DEV) * 0.02
            rank.view(name, rank.arenas[1]).copy_(full[p["r0"]:p["r1"], p["c0"]:p["c1"]])
        rank.arenas[0].copy_(rank.arenas[1])
    return ranks


def reshard(plan, old):
    """The new ranks with the old ones' states.  On more GPUs an exchange of the messages stands in between."""
    send = []
    for s, rank in enumerate(old):
        send.append(torch.empty(max(plan.send_layout(s)[3], 256), dtype=torch.uint8, device=DEV))
        etc.etc_pack(plan, s, rank.arenas, send[s])
    new = fresh_ranks(plan, etc.SIDE_DST, plan.D)
    for d, rank in enumerate(new):
        msgs = []
        for s in range(plan.S):
            counts, _, displs, _ = plan.send_layout(s)
            msgs.append(send[s].data_ptr() + int(displs[d]) if counts[d] else None)
        etc.etc_unpack(plan, d, msgs, rank.arenas)
    torch.cuda.current_stream().synchronize()  # the send buffers go away with this frame
    return new


def step(ranks, number, tokens, target):
    """One optimizer step (number counts from 1); returns the loss."""
    n, h = tokens.numel(), MODEL.hidden
    rows = torch.arange(n, device=DEV)
    positions = rows % LENGTH
    act = lambda: torch.empty(n, h, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    first, second = etc.Dropout(P, seed=number, call=0), etc.Dropout(P, seed=number, call=1)

    # forward: each token's row is on one rank, so the sum over ranks (an all-reduce) is exact
    summed = torch.zeros(n, h, dtype=torch.bfloat16, device=DEV)
    for rank in ranks:
        share = act()
        etc.etc_embed(tokens, rank.param("embed"), share, row0=rank.pieces["embed"]["r0"])
        summed += share
    x, y = act(), act()
    # replicated on all ranks: scale, positions and dropout, with the summed rows in the table's place
    etc.etc_embed(rows, summed, x, scale=SCALE, positions=positions, pos_table=ranks[0].param("pos_embed"),
                  dropout=first)
    bias = ranks[0].param("layers.0.proj.bias").view(-1)
    etc.etc_dropout(x, y, second, bias=bias, residual=x)
    error = y.float() - target
    loss = 0.5 * error.square().sum() / n

    # backward
    dy = (error / n).to(torch.bfloat16)
    dx = act()
    for rank in ranks:
        rank.grads.zero_()
    work = torch.empty(max(etc.etc_dropout_grad_bytes(n, h),
                           *(etc.etc_embed_grad_bytes(n, r.grad("embed").shape[0], h) for r in ranks),
                           etc.etc_embed_grad_bytes(n, MODEL.max_pos, h)), dtype=torch.uint8, device=DEV)
    for rank in ranks:
        etc.etc_dropout_grad(dy, dx, second, dbias=rank.grad("layers.0.proj.bias").view(-1), workspace=work)
        both = dx + dy  # through the epilogue's dropout and past it
        etc.etc_embed_grad(tokens, both, rank.grad("embed"), work, row0=rank.pieces["embed"]["r0"], scale=SCALE,
                           dropout=first)
        etc.etc_embed_grad(positions, both, rank.grad("pos_embed"), work, dropout=first)
        etc.etc_adam(rank.arenas, rank.grads, step=number, lr=LR, weight_decay=0.01)
    return loss


def train(change_after, steps=6):
    """(losses, the states at the end in the new configuration): a job that reshards after `change_after` steps."""
    plan = etc.etc_plan(MODEL, OLD, NEW, flags=etc.PLAN_SKETCH)
    ranks = fresh_ranks(plan, etc.SIDE_SRC, plan.S, seed=1)
    gen = torch.Generator(device=DEV).manual_seed(7)
    losses = []
    for number in range(1, steps + 1):
        tokens = torch.randint(0, MODEL.vocab, (SEQUENCES * LENGTH,), generator=gen, device=DEV)
        target = torch.randn(SEQUENCES * LENGTH, MODEL.hidden, generator=gen, device=DEV)
        losses.append(step(ranks, number, tokens, target))
        if number == change_after:
            ranks = reshard(plan, ranks)
    return [float(x) for x in losses], [r.arenas for r in ranks]


def main():
    moved, there = train(change_after=3)
    stayed, here = train(change_after=6)
    for number, (a, b) in enumerate(zip(moved, stayed), 1):
        print(f"step {number}: loss {a:.6f} (job on TP 4 from step 4 on), {b:.6f} (job on TP 2)")
    same = moved == stayed and all(torch.equal(x, y) for a, b in zip(there, here) for x, y in zip(a, b))
    print("the states are the same, bit for bit" if same else "THE STATES DIFFER")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
