"""Plain implementations in 64 bits of the operators around a block's
projections, from their definitions in include/etc.h, on the host, with numpy
alone; and bounds on what 32-bit arithmetic may be off.

As in op_ref.py, functions return (values, bound): `bound` is an absolute error
per element before the result is rounded to the output's type, from the unit
roundoff u = 2^-24 of 32-bit results.  What has to be equal bit for bit (the data
and scales of etc_store8, what etc_load8 reads) is worked out in the 32-bit
steps of the definition."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
TOP = {"i8": 127.0, "e4m3": 448.0}
LEAST = np.float32(2.0 ** -100)


def depth(cols):
    """Additions that a term of a row's sum passes at most: those of its lane
    (32 columns, or the row over 1024 lanes), 6 over the lanes, 16 over the wavefronts."""
    return max(32, -(-cols // 1024) + 8) + 6 + 16


# ---------------------------------------------------------------------------
# 8 bits

def e4m3_table():
    """The value of each of the 256 codes."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = np.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = -v if c >> 7 else v
    return out


E4M3 = e4m3_table()


def nearest_e4m3(v):
    """Codes of the e4m3 numbers nearest to v (|v| < 464), ties to the even code."""
    mags = E4M3[:127]  # 0 .. 448, ascending
    a = np.abs(v)
    hi = np.clip(np.searchsorted(mags, a), 1, 126)
    lo = hi - 1
    below, above = a - mags[lo], mags[hi] - a
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def groups(cols, group):
    return -(-cols // group) if group else 1


def store8(x, eight, group, col_scale=None):
    """(data as bytes [rows, cols], scales [rows, groups]) of fp32 x, in the definition's 32-bit steps."""
    x = np.asarray(x, np.float32)
    if col_scale is not None:
        x = x * np.asarray(col_scale, np.float32)[None, :]
    rows, cols = x.shape
    width = group or cols
    data, scale = np.zeros((rows, cols), np.uint8), np.zeros((rows, groups(cols, group)), np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        for g in range(scale.shape[1]):
            part = x[:, g * width:(g + 1) * width]
            a = np.abs(part).max(1, keepdims=True)
            fine = np.isfinite(a)
            a = np.maximum(np.where(fine, a, np.float32(0)), LEAST)
            top = np.float32(TOP[eight])
            factor = top / a
            if eight == "i8":  # the product is rounded once, to a whole number
                q = np.rint(part.astype(np.float64) * factor.astype(np.float64))
                code = np.where(fine, q, 0).astype(np.int64).astype(np.uint8)
            else:
                code = nearest_e4m3(np.where(fine, part * factor, np.float32(0)).astype(np.float64))
            data[:, g * width:(g + 1) * width] = np.where(fine, code, 0)
            scale[:, g] = np.where(fine, a / top, np.float32(np.nan))[:, 0]
    return data, scale


def values8(data, eight):
    """What the bytes stand for, unscaled."""
    return E4M3[data] if eight == "e4m3" else data.view(np.int8).astype(np.float64)


def load8(data, scale, eight, group):
    """fp32 values, rounded once."""
    cols = data.shape[1]
    wide = np.repeat(scale, group, 1)[:, :cols] if group else np.repeat(scale, cols, 1)
    return (values8(data, eight) * wide.astype(np.float64)).astype(np.float32)


# ---------------------------------------------------------------------------
# norm

def norm(x, weight, residual=None, eps=1e-6):
    """{sum, rstd, out}: (values, bound)."""
    x, w = x.astype(np.float64), weight.astype(np.float64)
    s = x if residual is None else x + residual.astype(np.float64)
    cols = x.shape[1]
    r = 1.0 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    # s and its square 3, the sum, 1 / cols and its product and eps 4; halved by the root, which adds 1; the quotient 1
    er = ((3 + depth(cols) + 4) / 2 + 2) * U
    y = s * r * w[None, :]
    return {"sum": (s, U * np.abs(s)), "rstd": (r[:, 0], er * r[:, 0]), "out": (y, (er + 4 * U) * np.abs(y))}


def check_norm8(data, scale, eight, want):
    """Whether 8-bit data and one scale a row are those of the norm `want` = (y,
    bound): the scale is that of the largest magnitude, and the data lie half a
    step from y at most, of which the bounds' share and 8 roundings are taken off."""
    y, bound = want
    a, top = np.abs(y).max(1), TOP[eight]
    off = np.divide(bound.max(1), np.maximum(a, 1e-300)) + 8 * U
    unit = np.maximum(a, float(LEAST)) / top
    assert np.all(np.abs(scale - unit) <= off * unit), "scale"
    v = y / unit[:, None]
    q = values8(data, eight)
    # e4m3: half a step is 2^-4 of the value, or 2^-10 among the smallest
    half = np.full_like(v, 0.5) if eight == "i8" else np.maximum(np.abs(v) * 2.0 ** -4, 2.0 ** -10)
    far = np.abs(q - v) - half - np.maximum(np.abs(v), np.abs(q)) * 2 * off[:, None]
    assert np.all(far <= 0), ("data", float(far.max()), np.argwhere(far > 0)[:3].tolist())
    # a row's largest element is the type's
    rows = np.arange(len(a))
    big = np.abs(q)[rows, np.abs(y).argmax(1)]
    assert np.all((big == top) | (a < float(LEAST))), "largest"


def norm_grad(grad, x, weight, rstd, dsum=None, before=None, accumulate=False, kept=False):
    """{dx, dweight}: (values, bound); rstd: as given.  kept: x was worked out from 8 bits in 32."""
    g, w, x = grad.astype(np.float64), weight.astype(np.float64)[None, :], x.astype(np.float64)
    r, cols = rstd.astype(np.float64)[:, None], grad.shape[1]
    n, dn = x * r, g * w
    en = (2 if kept else 1) * U  # n: the scale times r, and the data
    mean = (dn * n).mean(1, keepdims=True)
    # each term: n, dn and their product; the sum; 1 / cols and its product
    emean = (en + (2 + depth(cols) + 2) * U) * np.abs(dn * n).mean(1, keepdims=True)
    d = np.zeros_like(g) if dsum is None else dsum.astype(np.float64)
    dx = d + r * (dn - n * mean)
    size = r * (np.abs(dn) + np.abs(n * mean))
    bound = (en + 5 * U) * size + r * np.abs(n) * emean + U * np.abs(dx)
    out = {"dx": (dx, bound)}
    if before is not None:
        total = (g * n).sum(0)
        size = np.abs(g * n).sum(0)
        out["dweight"] = (total + before if accumulate else total,
                          (en + (grad.shape[0] + 2) * U) * size + (2 * U * (np.abs(total) + np.abs(before)) if accumulate else 0.0))
    return out


# ---------------------------------------------------------------------------
# products and rotations

def matmul8(x, w, sx=None, sw=None, bias=None):
    """(values, bound); x and w int8."""
    acc = x.astype(np.int64) @ w.astype(np.int64).T
    assert not acc.size or np.abs(acc).max() < 1 << 31
    y = acc.astype(np.float64)
    if sx is not None:
        y = y * sx.astype(np.float64)[:, None]
    if sw is not None:
        y = y * sw.astype(np.float64)[None, :]
    bound = 3 * U * np.abs(y)  # the sum to 32 bits, two products
    if bias is not None:
        y = y + bias.astype(np.float64)[None, :]
        bound = bound + U * np.abs(y) * (1 + U)
    return y, bound + U * bound


def frequencies(dim, base=10000.0, scaling=None, factor=1.0, length=0.0, low=1.0, high=32.0):
    j = np.arange(dim // 2)
    if scaling == "base":
        base = base * factor ** (dim / (dim - 2))
    f = base ** (-2.0 * j / dim)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        u = np.clip((length * f / (2 * np.pi) - low) / (high - low), 0, 1)
        f = f * (u + (1 - u) / factor)
    return f


def rotary(x, positions, freq, head_dim, layout="half", scale=1.0, backward=False):
    """(values, bound)."""
    rows, cols = x.shape
    p = len(freq)
    h = x.astype(np.float64).reshape(rows, cols // head_dim, head_dim)
    angle = np.asarray(positions, np.float64)[:, None] * freq[None, :]
    c, s = (scale * f(angle)[:, None, :] for f in (np.cos, np.sin))
    s = -s if backward else s
    at = (slice(0, p), slice(p, 2 * p)) if layout == "half" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    a, b = h[..., at[0]], h[..., at[1]]
    out, bound = h.copy(), np.zeros_like(h)
    out[..., at[0]], out[..., at[1]] = a * c - b * s, b * c + a * s
    # the angle: three roundings of 64 bits here and there, and what is left of a turn rounded to 32 bits (2^-26 of a
    # turn); sine and cosine within 2 units of 2^-24, times scale 2, a product and the sum
    off = np.abs(angle)[:, None, :] * 6 * 2.0 ** -53 + 2 * np.pi * 2.0 ** -26 + 2 * 2.0 ** -23
    e = abs(scale) * (off + 4 * U) * (np.abs(a) + np.abs(b))
    bound[..., at[0]], bound[..., at[1]] = e, e
    return out.reshape(rows, cols), bound.reshape(rows, cols)
