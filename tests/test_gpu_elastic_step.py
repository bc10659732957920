"""The example that runs the operators together: a job that changes from TP 2
to TP 4 between two steps ends in the states of one that stays, bit for bit,
and what it trains improves."""
import importlib.util
import os

import pytest
import torch

from gpu_util import say

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "elastic_input_stage.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("elastic_input_stage", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_resharded_job_equals_the_one_that_stays(example):
    say("example: TP 2 -> TP 4 after step 3 of 6, and after step 6")
    moved, there = example.train(change_after=3)
    stayed, here = example.train(change_after=6)
    assert moved == stayed and len(there) == len(here) == 4
    for a, b in zip(there, here):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
    for arenas in there:
        assert bool(arenas[3].any()) and torch.equal(arenas[0], arenas[1].to(torch.bfloat16))
        assert all(bool(torch.isfinite(x).all()) for x in arenas)


def test_other_seed_gives_other_states(example):
    """The comparison above would see a difference: another number of steps does."""
    say("example: five steps")
    _, five = example.train(change_after=5, steps=5)
    _, six = example.train(change_after=6, steps=6)
    assert any(not torch.equal(x, y) for a, b in zip(five, six) for x, y in zip(a, b))


def test_it_learns(example):
    """The same batch again and again: the loss falls."""
    say("example: one batch, 30 steps")
    plan = example.etc.etc_plan(example.MODEL, example.OLD, example.NEW)
    ranks = example.fresh_ranks(plan, example.etc.SIDE_SRC, plan.S, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(7)
    tokens = torch.randint(0, example.MODEL.vocab, (512,), generator=gen, device="cuda")
    target = torch.randn(512, example.MODEL.hidden, generator=gen, device="cuda")
    losses = [float(example.step(ranks, k, tokens, target)) for k in range(1, 31)]
    assert losses[-1] < 0.95 * losses[0], losses
