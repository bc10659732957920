"""Cases of the norm's weight gradient that have one right answer: gradients and
inputs are whole numbers, 1 / rms is 1 or 2, and each column's terms are of one
sign, so that every sum of terms, in any order, is a whole number below 2^24, which
32 bits hold exactly, and a sum that lacks any of its terms, or has one twice, is
another number."""
from __future__ import annotations

import numpy as np

LIMIT = 1 << 24

# rows, cols, dtype, x kept in, its group
DWEIGHT = [
    # one launch, up to 1024 rows
    (1, 8, "bf16", None, 0), (2, 1, "f32", None, 0), (300, 4096, "bf16", "i8", 128), (513, 681, "f32", None, 0), (1021, 681, "f32", None, 0),
    (1024, 100, "bf16", "e4m3", 32), (1000, 2048, "bf16", None, 0), (128, 16384, "bf16", None, 0),
    # rows of several wavefronts, one block a lane and two
    (1025, 681, "bf16", None, 0), (8192, 681, "bf16", "i8", 256), (4099, 1033, "f32", None, 0), (1025, 8192, "bf16", "e4m3", 64),
    (129, 16384, "bf16", None, 0), (1100, 5001, "f32", "i8", 0),
    # rows that share wavefronts: none, 4 and 16 of which join their sums
    (1030, 255, "bf16", None, 0), (4099, 256, "bf16", None, 0), (17000, 512, "bf16", None, 0), (17001, 257, "bf16", None, 0),
    (16384, 500, "bf16", "e4m3", 64), (5003, 128, "bf16", None, 0), (33000, 128, "bf16", None, 0), (70001, 128, "bf16", None, 0),
    (70003, 121, "bf16", "i8", 32), (33000, 8, "bf16", None, 0), (262144, 16, "bf16", None, 0), (1048577, 5, "f32", None, 0),
    (4100, 256, "f32", None, 0), (17003, 129, "f32", None, 0), (70001, 63, "f32", None, 0), (9001, 17, "f32", "i8", 32),
    # rows of less than a block, and rows that registers do not hold
    (70001, 3, "f32", None, 0), (5000, 7, "bf16", None, 0), (600, 20001, "f32", None, 0), (300, 33000, "bf16", "i8", 0),
]


def dweight_case(case):
    """(grad, x's whole numbers, x's scales or None, 1 / rms, what dweight holds before)."""
    rows, cols, _, kept, group = case
    rng = np.random.default_rng([rows, cols])
    grad, x = (rng.integers(1, 4, (rows, cols), dtype=np.int8) for _ in range(2))
    grad *= rng.choice(np.array((-1, 1), np.int8), cols)[None, :]
    x *= rng.choice(np.array((-1, 1), np.int8), cols)[None, :]
    scale = None
    if kept:
        scale = rng.integers(1, 3, (rows, -(-cols // group) if group else 1)).astype(np.float32)
    r = rng.integers(1, 3, rows).astype(np.float32) if rows < 1 << 18 else np.ones(rows, np.float32)
    return grad, x, scale, r, rng.integers(-3, 4, cols)


def wide(x, scale, group):
    """x times its scales."""
    if scale is None:
        return x.astype(np.int32)
    s = np.repeat(scale.astype(np.int32), group or x.shape[1], 1)[:, :x.shape[1]]
    return x * s


def dweight_sums(grad, x, scale, group, r):
    """The sums over rows of grad * x * r."""
    terms = wide(x, scale, group) * grad * r.astype(np.int32)[:, None]
    assert np.abs(terms).sum(0, dtype=np.int64).max(initial=0) + 3 < LIMIT
    return terms.sum(0, dtype=np.int64)
