"""Cases of the operators' sums that have one right answer: whole numbers, none
of them zero, and scales that are powers of two, so that every sum of terms, in
any order, is a whole number below 2^24, which 32 bits hold exactly.  A sum that
lacks a term, or has one twice, is another number."""
from __future__ import annotations

import numpy as np

import op_ref

LIMIT = 1 << 24

# tokens, cols, rows, ids, dropout's p (0 or 1/2, which scales by 2), dtype
GRAD = [
    (512, 40, 5, "same", 0.0, "bf16"),
    (512, 264, 40, "log", 0.5, "f32"),
    (1024, 24, 7, "log", 0.0, "bf16"),
    (1025, 24, 3000, "log", 0.0, "bf16"),
    (2048, 17, 9, "log", 0.5, "f32"),
    (2049, 64, 9, "same", 0.0, "bf16"),
    (4096, 8, 1024, "fours", 0.0, "bf16"),
    (5003, 1032, 11, "log", 0.5, "bf16"),
    (16384, 2048, 5000, "log", 0.0, "bf16"),
    (16385, 24, 8000, "distinct", 0.0, "f32"),
    (33000, 12, 9, "same", 0.0, "f32"),
    (33000, 600, 9, "same", 0.5, "bf16"),
    (70001, 256, 300, "log", 0.5, "bf16"),
    (70001, 9, 70001, "distinct", 0.0, "bf16"),
    (300007, 33, 2, "log", 0.0, "f32"),
    (1048577, 1, 3, "log", 0.0, "f32"),
    (1100003, 8, 50000, "log", 0.0, "bf16"),
]

# rows, cols, p, dtype
BIAS = [(1, 24, 0.0, "bf16"), (1024, 75, 0.5, "bf16"), (1024, 512, 0.0, "f32"), (1025, 75, 0.0, "bf16"), (5000, 40, 0.0, "f32"),
        (9001, 264, 0.0, "bf16"), (9001, 264, 0.5, "f32"), (70001, 33, 0.5, "bf16"), (4097, 8192, 0.0, "bf16"),
        (1048577, 5, 0.0, "f32")]


def whole(rng, *shape):
    """-3 .. 3 without 0."""
    x = rng.integers(1, 4, shape, dtype=np.int64)
    return np.where(rng.random(shape) < 0.5, -x, x)


def ids_of(rng, n, rows, kind):
    """Ids of a table of `rows` rows, and with "log" some outside it."""
    if kind == "same":
        return np.full(n, rows // 2, np.int64)
    if kind == "distinct":
        return rng.permutation(np.arange(n, dtype=np.int64)) % rows
    if kind == "fours":  # runs of four, which end where chunks of four do
        return rng.permutation(np.arange(n, dtype=np.int64) // 4 % rows)
    v = np.exp(rng.random(n) * np.log(rows + 1)).astype(np.int64) - 1
    v[::11] = -1
    v[5::977] = rows
    return v


def _kept(rows, cols, drop):
    if not op_ref.limit(drop[0]):
        return np.int64(1)
    kept, scale = op_ref.mask(rows, cols, *drop)
    assert scale == 2.0
    return kept.astype(np.int64) * 2


def grad_case(case):
    """(ids, gradients, what the table's gradient holds before, dropout); scale is 4."""
    n, cols, rows, kind, p, _ = case
    rng = np.random.default_rng([n, cols, rows])
    return ids_of(rng, n, rows, kind), whole(rng, n, cols), whole(rng, rows, cols), (p, 5, 1, 3)


def grad_sums(v, g, before, drop):
    """4 * the sums of each row's gradients, and added to `before`; every one below the limit."""
    rows, cols = before.shape
    g = g * _kept(*g.shape, drop)
    held = np.flatnonzero((v >= 0) & (v < rows))
    held = held[np.argsort(v[held], kind="stable")]
    out = np.zeros((rows, cols), np.int64)
    if held.size:
        first = np.flatnonzero(np.diff(v[held], prepend=-1))
        out[v[held][first]] = np.add.reduceat(g[held], first, axis=0)
        assert np.add.reduceat(np.abs(g[held]), first, axis=0).max() * 4 + 3 < LIMIT
    return out * 4, out * 4 + before


def bias_case(case):
    rows, cols, p, _ = case
    rng = np.random.default_rng([rows, cols])
    return whole(rng, rows, cols), whole(rng, cols), (p, 6, 2, (1 << 32) - 5)


def bias_sums(g, before, drop):
    g = g * _kept(*g.shape, drop)
    assert np.abs(g).sum(0).max() + 3 < LIMIT
    return g, g.sum(0), g.sum(0) + before
