"""Plain implementations in 64 bits of the operators of a training step, from
their definitions in include/etc.h, on the host, with numpy alone; and bounds
on what 32-bit sums may be off.

Each function returns (values, bound): `bound` is an absolute error per
element before the result is rounded to the output's type, from the unit
roundoff u = 2^-24 of 32-bit results.  Rounding is monotone, so a bf16 output
has to lie between the roundings of value - bound and value + bound."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def philox(counter, key):
    """Philox4x32-10 of counters [4][...] and a 2-word key, in Python's terms."""
    c = [np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF) for x in counter]
    k0, k1 = int(key[0]), int(key[1])
    w = np.uint64(32)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        hp, lp, hq, lq = p >> w, p & np.uint64(0xFFFFFFFF), q >> w, q & np.uint64(0xFFFFFFFF)
        c = [hq ^ c[1] ^ np.uint64(k0), lq, hp ^ c[3] ^ np.uint64(k1), lp]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def limit(p):
    return int(np.floor(65536.0 * p + 0.5))


def mask(rows, cols, p, seed, call=0, row0=0):
    """(kept [rows, cols], scale of what is kept)."""
    t = limit(p)
    blocks = (cols + 7) // 8
    r = np.array([row0 + i for i in range(rows)], np.uint64)[:, None]
    b = np.arange(blocks, dtype=np.uint64)[None, :]
    z = np.zeros((rows, blocks), np.uint64)
    c = philox((z + b, z + (r & np.uint64(0xFFFFFFFF)), z + (r >> np.uint64(32)), z + np.uint64(call)),
               (seed & 0xFFFFFFFF, seed >> 32))
    u = np.empty((rows, blocks, 8), np.int64)
    for j in range(4):
        u[:, :, 2 * j] = (c[j] & np.uint64(0xFFFF)).astype(np.int64)
        u[:, :, 2 * j + 1] = (c[j] >> np.uint64(16)).astype(np.int64)
    kept = u.reshape(rows, blocks * 8)[:, :cols] >= t
    return kept, 65536.0 / (65536 - t) if t < 65536 else 0.0


def _drop(x, drop):
    """(dropped x, scale): drop is None or (p, seed, call, row0)."""
    if drop is None or limit(drop[0]) == 0:
        return x, 1.0, np.ones(x.shape, bool)
    kept, s = mask(*x.shape, *drop)
    return np.where(kept, np.where(kept, x, 0.0) * s, 0.0), s, kept


def embed(ids, table, row0=0, scale=1.0, positions=None, pos_table=None, drop=None):
    ids = [int(v) - row0 for v in ids]
    x = np.zeros((len(ids), table.shape[1]))
    for i, k in enumerate(ids):
        if 0 <= k < table.shape[0]:
            x[i] = table[k].astype(np.float64) * scale
    size = np.abs(x)
    if positions is not None:
        for i, q in enumerate(positions):
            if 0 <= int(q) < pos_table.shape[0]:
                x[i] += pos_table[int(q)]
                size[i] += np.abs(pos_table[int(q)])
    x, s, kept = _drop(x, drop)
    # scale and s are rounded once each, and up to three products and sums
    bound = 6 * U * s * np.where(kept, size, 0.0)
    return x, bound


def embed_grad(ids, grad, before, row0=0, scale=1.0, drop=None, accumulate=False):
    g, _, _ = _drop(grad.astype(np.float64), drop)
    d, size, count = np.zeros(before.shape), np.zeros(before.shape), np.zeros(before.shape[0])
    k = np.asarray(ids, np.int64) - row0
    held = (k >= 0) & (k < before.shape[0])
    np.add.at(d, k[held], g[held])
    np.add.at(size, k[held], np.abs(g[held]))
    np.add.at(count, k[held], 1)
    d *= scale
    size *= abs(scale)
    out = d + before if accumulate else d
    # n terms in any order: n - 1 sums; the kept scale (rounded, multiplied), scale (the same) and the last sum
    return out, U * ((count[:, None] + 5) * size + (np.abs(out) + np.abs(before) if accumulate else 0.0))


def dropout(x, bias=None, residual=None, drop=None):
    y = x.astype(np.float64) + (0.0 if bias is None else bias.astype(np.float64)[None, :])
    size = np.abs(x.astype(np.float64)) + (0.0 if bias is None else np.abs(bias.astype(np.float64))[None, :])
    y, s, kept = _drop(y, drop)
    size = np.where(kept, size, 0.0) * s
    if residual is not None:
        y = y + residual.astype(np.float64)
        size = size + np.abs(residual.astype(np.float64))
    bound = 5 * U * size
    return y, bound


def dropout_grad(grad, before=None, drop=None, accumulate=False):
    g, _, _ = _drop(grad.astype(np.float64), drop)
    dx = (g, 3 * U * np.abs(g))
    if before is None:
        return dx
    d = g.sum(0)
    total = d + before if accumulate else d
    bound = U * ((grad.shape[0] + 4) * np.abs(g).sum(0) + (np.abs(total) + np.abs(before) if accumulate else 0.0))
    return dx, (total, bound)


def adam(master, m, v, grad, step, lr, beta1, beta2, eps, weight_decay, scale=1.0):
    """{param, master, m, v}: (values, bound)."""
    w, m0, v0, g = (x.astype(np.float64) for x in (master, m, v, grad))
    g = g * scale
    m1 = beta1 * m0 + (1 - beta1) * g
    v1 = beta2 * v0 + (1 - beta2) * g * g
    # each term: its factor rounded, up to three products, and the sum
    m_size = beta1 * np.abs(m0) + (1 - beta1) * np.abs(g)
    mb, vb = 5 * U * m_size, 6 * U * v1
    c1, c2 = 1 - beta1 ** step, 1 - beta2 ** step
    den = np.sqrt(v1 / c2) + eps
    with np.errstate(divide="ignore", invalid="ignore"):
        update = lr * (m1 / c1) / den
        size = abs(lr) * (m_size / c1) / den
    out = w - (update + lr * weight_decay * w)
    # the quotient: 5 from m, 5 from the root (half of 6 and 2, and its own), eps and the sum 2, lr / c1 and two operations 3
    bound = U * (16 * size + 4 * abs(lr * weight_decay) * np.abs(w) + 2 * (np.abs(out) + size))
    return {"master": (out, bound), "m": (m1, mb), "v": (v1, vb), "param": (out, bound)}
