"""The operators of a training step on the GPU, through the C ABI, against
plain implementations in 64 bits (op_ref.py): embedding lookup and gradient,
dropout and its backward, Adam.  Sizes from nothing over one to odd ones, ids
outside the table, rows further apart than they are long, offsets past 32 bits, NaN and
infinities in dropped places, accumulation, repeated and captured calls."""
import numpy as np
import pytest
import torch

import op_ref
from gpu_util import DEV, say
from paper_2607_04749_amd import etc

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CANARY = -7.0  # in the elements between the rows of an output


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def rand(rng, rows, cols, dtype, std=1.0, more=0, shift=0):
    """(device view [rows, cols], its values in numpy): rows `more` elements
    further apart than they are long, `shift` elements into the buffer."""
    x = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32) * std).to(DT[dtype])
    full = torch.full((shift + rows * (cols + more) + 8,), CANARY, dtype=DT[dtype], device=DEV)
    view = full[shift:shift + rows * (cols + more)].view(rows, cols + more)[:, :cols]
    view.copy_(x.to(DEV))
    return view, x.float().numpy(), full


def blank(rows, cols, dtype, more=0, shift=0):
    full = torch.full((shift + rows * (cols + more) + 8,), CANARY, dtype=DT[dtype], device=DEV)
    return full[shift:shift + rows * (cols + more)].view(rows, cols + more)[:, :cols], full


def untouched(full, view):
    """The elements of a buffer outside the view still hold the canary."""
    outside = torch.ones_like(full, dtype=torch.bool)
    at = torch.as_strided(outside, view.shape, view.stride(), view.storage_offset())
    at.fill_(False)
    return bool((full[outside] == CANARY).all())


def close(got, want, what):
    """Within the bound of the value; a bf16 result between the roundings of the bound's ends."""
    value, bound = want
    low, high = value - bound - 1e-300, value + bound + 1e-300
    if got.dtype == torch.bfloat16:
        low, high = (torch.from_numpy(x).float().to(torch.bfloat16).double().numpy() for x in (low, high))
    got = got.double().cpu().numpy()
    assert got.shape == value.shape, what
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                           got[bad][:3], value[bad][:3], bound[bad][:3])


def workspace(nbytes):
    """Exactly the bytes asked for, before a canary, filled with what is no valid content."""
    full = torch.full((nbytes + 512,), 0xEE, dtype=torch.uint8, device=DEV)
    return full[:nbytes], full[nbytes:]


# ---------------------------------------------------------------------------
# embedding

def ids_of(rng, n, vocab, kind="log"):
    if kind == "log":  # frequent ids low
        v = np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64) - 1
    elif kind == "same":
        v = np.full(n, vocab // 2, np.int64)
    elif kind == "outside":
        v = np.where(rng.random(n) < 0.5, -1 - rng.integers(0, 5, n), vocab + rng.integers(0, 5, n))
    elif kind == "distinct":
        v = np.arange(n, dtype=np.int64) % vocab
    return v


EMBED = [
    # tokens, cols, vocab, rows, row0, pos, p, table, out, ids, more, shift
    (1, 8, 16, 16, 0, 0, 0.0, "bf16", "bf16", "int64", 0, 0),
    (1, 4096, 100, 100, 0, 0, 0.0, "bf16", "bf16", "int32", 0, 0),
    (1, 1, 1, 1, 0, 0, 0.0, "f32", "f32", "int64", 0, 0),
    (0, 64, 10, 10, 0, 0, 0.1, "bf16", "bf16", "int64", 0, 0),
    (7, 0, 10, 10, 0, 0, 0.1, "bf16", "bf16", "int64", 0, 0),
    (5, 24, 8, 0, 3, 0, 0.0, "bf16", "bf16", "int64", 0, 0),
    (67, 597, 300, 100, 100, 0, 0.0, "bf16", "bf16", "int64", 0, 0),
    (129, 681, 300, 100, 200, 17, 0.1, "bf16", "bf16", "int32", 3, 1),
    (33, 504, 64, 64, 0, 128, 0.5, "f32", "f32", "int64", 0, 3),
    (40, 2048, 64, 32, 32, 5, 0.25, "bf16", "f32", "int32", 8, 0),
    (40, 2047, 64, 32, 0, 5, 0.0, "f32", "bf16", "int64", 1, 5),
    (1000, 256, 1024, 256, 512, 128, 0.1, "bf16", "bf16", "int64", 0, 0),
    (9, 15, 20, 20, 0, 4, 1.0, "bf16", "f32", "int64", 0, 0),
    (300, 7, 40, 40, 0, 0, 0.3, "f32", "bf16", "int64", 2, 1),
    # as many blocks as make a lane take two rows; an odd number of rows
    (65537, 128, 300, 100, 100, 0, 0.1, "bf16", "bf16", "int64", 0, 0),
    (65539, 121, 300, 100, 100, 17, 0.1, "bf16", "bf16", "int32", 3, 1),
    (32769, 127, 64, 64, 0, 33, 0.5, "f32", "f32", "int64", 0, 0),
    (65537, 121, 8, 0, 3, 5, 0.1, "bf16", "bf16", "int64", 0, 0),
] + [
    # every kernel: types, whole blocks or not, dropout or not, one row a lane or two
    (tokens, cols, 40, 30, 5, 6, p, table, out, "int64", 1, 1)
    for table in ("bf16", "f32") for out in ("bf16", "f32")
    for tokens, cols, p in ((37, 40, 0.0), (37, 39, 0.0), (37, 40, 0.1), (37, 39, 0.1), (32771, 256, 0.1), (32771, 255, 0.1))
]


@pytest.mark.parametrize("case", EMBED, ids=lambda c: "-".join(map(str, c)))
def test_embed(case):
    tokens, cols, vocab, rows, row0, pos, p, table, out, ids, more, shift = case
    say("embed", case)
    rng = np.random.default_rng(list(case[:6]))
    v = ids_of(rng, tokens, vocab)
    v[::7] = -1
    w, wn, _ = rand(rng, rows, cols, table, more=more, shift=shift)
    o, full = blank(tokens, cols, out, more=more, shift=shift)
    d = (p, 0x1234567890ABCDEF, 3, 11)
    kw = {}
    ref = dict(row0=row0, scale=1.75, drop=d)
    if pos:
        pw, pn, _ = rand(rng, pos, cols, table)
        q = np.arange(tokens) % (pos + 1)  # one past the table: contributes nothing
        kw = dict(positions=torch.from_numpy(q).to(getattr(torch, ids)).to(DEV), pos_table=pw)
        ref.update(positions=q, pos_table=pn)
    etc.etc_embed(torch.from_numpy(v).to(getattr(torch, ids)).to(DEV), w, o, row0=row0, scale=1.75,
                  dropout=etc.Dropout(*d), **kw)
    torch.cuda.synchronize()
    close(o, op_ref.embed(v, wn, **ref), case)
    assert untouched(full, o)


@pytest.mark.parametrize("tokens", (40, 70001))
def test_embed_reads_no_row_for_ids_outside(tokens):
    """Whatever the tables hold, infinities and NaN among it, ids and positions
    outside them contribute zeros."""
    say("embed: ids outside", tokens)
    w = torch.full((3, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    q = torch.full((2, 128), float("inf"), dtype=torch.bfloat16, device=DEV)
    v = torch.arange(tokens, device=DEV) % 2 * 8 - 5  # -5 and 3, of a table of 0 .. 2
    for kw in ({}, dict(positions=v, pos_table=q), dict(positions=v, pos_table=q[:0])):
        o = torch.ones(tokens, 128, dtype=torch.bfloat16, device=DEV)
        etc.etc_embed(v, w, o, dropout=etc.Dropout(0.2, 1), **kw)
        assert not bool(o.any()) and not bool(o.isnan().any())


def test_embed_without_dropout_is_exact():
    """Scale 1 and no positions: the rows themselves, and exact zeros outside."""
    say("embed: copies")
    rng = np.random.default_rng(5)
    w, _, _ = rand(rng, 50, 333, "bf16")
    v = torch.from_numpy(ids_of(rng, 200, 80)).to(DEV)
    o, _ = blank(200, 333, "bf16")
    etc.etc_embed(v, w, o, row0=10)
    k = v - 10
    held = (k >= 0) & (k < 50)
    want = torch.where(held[:, None], w[k.clamp(0, 49)], torch.zeros((), dtype=torch.bfloat16, device=DEV))
    assert torch.equal(o, want)


def test_embed_empty_position_table():
    """A position table of no rows contributes nothing, as positions past one do."""
    say("embed: empty position table")
    rng = np.random.default_rng(7)
    w, wn, _ = rand(rng, 6, 40, "bf16")
    v = torch.arange(6, device=DEV)
    o, _ = blank(6, 40, "f32")
    etc.etc_embed(v, w, o, positions=v, pos_table=w[:0])
    close(o, op_ref.embed(range(6), wn), "empty")
    etc.etc_embed(v[:0], w, o[:0], positions=v[:0], pos_table=w)


def test_embed_extreme_ids():
    """Ids at the ends of 64 and 32 bits are outside, whatever row0 is."""
    say("embed: extreme ids")
    rng = np.random.default_rng(6)
    w, wn, _ = rand(rng, 4, 16, "f32")
    for row0 in (0, 5, (1 << 62), -3):
        v = np.array([-(1 << 63), (1 << 63) - 1, -1, row0, row0 + 3, row0 + 4, row0 - 1], np.int64)
        o, _ = blank(len(v), 16, "f32")
        etc.etc_embed(torch.from_numpy(v).to(DEV), w, o, row0=row0)
        close(o, op_ref.embed(v, wn, row0=row0), row0)
    v = np.array([-(1 << 31), (1 << 31) - 1, 2], np.int32)
    o, _ = blank(len(v), 16, "f32")
    etc.etc_embed(torch.from_numpy(v).to(DEV), w, o, row0=1)
    close(o, op_ref.embed(v, wn, row0=1), "int32")


def test_shards_add_up():
    """The lookups of the shares of a vocabulary, added, are the whole one's, bit for bit."""
    say("embed: shards")
    rng = np.random.default_rng(8)
    w, _, _ = rand(rng, 120, 264, "bf16")
    v = torch.from_numpy(ids_of(rng, 500, 120)).to(DEV)
    whole, _ = blank(500, 264, "bf16")
    etc.etc_embed(v, w, whole, scale=3.0)
    for tp in (2, 3, 4):
        total = torch.zeros_like(whole)
        for r in range(tp):
            n = 120 // tp
            part, _ = blank(500, 264, "bf16")
            etc.etc_embed(v, w[r * n:(r + 1) * n], part, row0=r * n, scale=3.0)
            total += part
        assert torch.equal(total, whole)


GRAD = [
    # tokens, cols, vocab, rows, row0, p, dtype, ids, kind, more, shift
    (1, 8, 16, 16, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (1, 1, 1, 1, 0, 0.0, "f32", "int32", "log", 0, 0),
    (0, 40, 16, 16, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (9, 40, 16, 0, 16, 0.1, "bf16", "int64", "log", 0, 0),
    (9, 0, 16, 16, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (64, 256, 32, 32, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (65, 24, 5000, 5000, 0, 0.0, "f32", "int64", "distinct", 0, 0),
    (127, 681, 300, 100, 100, 0.1, "bf16", "int32", "log", 3, 1),
    (128, 597, 300, 100, 0, 0.0, "f32", "int64", "log", 1, 3),
    (513, 504, 64, 64, 0, 0.5, "f32", "int64", "log", 0, 0),
    (1000, 33, 1024, 256, 0, 0.25, "bf16", "int32", "log", 0, 0),
    (2049, 520, 3, 3, 0, 0.0, "bf16", "int64", "log", 8, 0),
    (3000, 64, 100, 100, 0, 0.1, "bf16", "int64", "same", 0, 0),
    (700, 72, 100, 100, 0, 0.1, "bf16", "int64", "outside", 0, 0),
    (4097, 40, 70000, 70000, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (8191, 16, 2000, 1000, 0, 0.0, "bf16", "int32", "log", 0, 0),
    (8193, 17, 2000, 1000, 500, 0.1, "f32", "int64", "log", 0, 0),
    (20000, 24, 300, 300, 0, 0.0, "f32", "int64", "log", 0, 0),
    (20011, 8, 140000, 140000, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (33000, 12, 9, 9, 0, 0.0, "f32", "int64", "same", 0, 0),
    (50, 9000, 40, 40, 0, 0.1, "bf16", "int64", "log", 0, 0),
    # around the sizes where the way of ordering changes
    (255, 40, 33, 33, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (256, 1032, 17, 17, 0, 0.0, "f32", "int32", "log", 0, 0),
    (256, 24, 5, 5, 0, 0.0, "bf16", "int64", "same", 0, 0),
    (257, 40, 33, 33, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (511, 24, 5000, 5000, 0, 0.0, "bf16", "int64", "distinct", 0, 0),
    (512, 2048, 300, 300, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (512, 2056, 300, 300, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (512, 24, 5, 5, 0, 0.0, "bf16", "int64", "same", 0, 0),
    (513, 24, 5000, 5000, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (128, 8192, 40, 40, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (129, 8192, 40, 40, 0, 0.1, "bf16", "int64", "log", 0, 0),
    (1024, 16, 900, 900, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (1025, 16, 900, 900, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (2048, 16, 900, 900, 0, 0.0, "bf16", "int32", "log", 0, 0),
    (2049, 16, 900, 900, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (2048, 16, 9, 9, 0, 0.0, "bf16", "int64", "same", 0, 0),
    # more columns than a launch for few takes, and one chunk of tokens
    (1, 530001, 2, 2, 0, 0.0, "f32", "int64", "log", 0, 0),
    (3, 200003, 4, 4, 0, 0.1, "f32", "int64", "same", 0, 0),
    (16384, 8, 900, 900, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (16385, 8, 900, 900, 0, 0.0, "bf16", "int64", "log", 0, 0),
    (40000, 9, 50000, 50000, 0, 0.1, "f32", "int32", "distinct", 0, 0),
    # every kernel: types, whole blocks or not, dropout or not
    (200, 33, 50, 40, 5, 0.0, "bf16", "int64", "log", 1, 1),
    (200, 64, 50, 40, 5, 0.1, "f32", "int64", "log", 0, 0),
    (200, 63, 50, 40, 5, 0.1, "f32", "int64", "log", 3, 1),
    (700, 33, 60, 50, 5, 0.0, "bf16", "int64", "log", 1, 1),
    # three levels of merging
    (1100003, 3, 60000, 50000, 100, 0.0, "f32", "int64", "log", 0, 0),
    (1048577, 1, 3, 3, 0, 0.0, "f32", "int64", "log", 0, 0),
]


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("case", GRAD, ids=lambda c: "-".join(map(str, c)))
def test_embed_grad(case, accumulate):
    tokens, cols, vocab, rows, row0, p, dtype, ids, kind, more, shift = case
    say("embed_grad", case, accumulate)
    rng = np.random.default_rng(list(case[:5]))
    v = ids_of(rng, tokens, vocab, kind)
    if kind == "log":
        v[::9] = -1
    g, gn, _ = rand(rng, tokens, cols, dtype, more=more, shift=shift)
    dt, before, full = rand(rng, rows, cols, "f32", more=more, shift=shift)
    d = (p, 77, 1, 1 << 33)
    ws, end = workspace(etc.etc_embed_grad_bytes(tokens, rows, cols))
    t = torch.from_numpy(v).to(getattr(torch, ids)).to(DEV)
    etc.etc_embed_grad(t, g, dt, ws, row0=row0, scale=0.75, dropout=etc.Dropout(*d), accumulate=accumulate)
    torch.cuda.synchronize()
    close(dt, op_ref.embed_grad(v, gn, before, row0, 0.75, d, accumulate), case)
    assert untouched(full, dt) and bool((end == 0xEE).all())
    if accumulate:  # rows of no token keep their bits
        none = np.setdiff1d(np.arange(rows), v - row0)
        assert np.array_equal(dt.cpu().numpy()[none], before[none])


@pytest.mark.parametrize("tokens", (700, 9000))
def test_embed_grad_repeats_to_the_bit(tokens):
    """The same call gives the same bits, on a workspace that other calls
    left behind, and on one that is larger than it needs."""
    say("embed_grad: repeated", tokens)
    rng = np.random.default_rng(9)
    v = torch.from_numpy(ids_of(rng, tokens, 50)).to(DEV)
    g, _, _ = rand(rng, tokens, 200, "f32")
    n = etc.etc_embed_grad_bytes(tokens, 50, 200)
    ws = torch.empty(n + 4096, dtype=torch.uint8, device=DEV)
    first = None
    for k in range(4):
        ws.random_(0, 256)
        dt = torch.empty(50, 200, device=DEV)
        etc.etc_embed_grad(v, g, dt, ws, dropout=etc.Dropout(0.1, 5))
        first = dt if first is None else first
        assert torch.equal(dt, first)


def test_embed_grad_against_differences():
    """The lookup is linear in the table: the gradient of sum(c * out) is the
    change of that sum when one element of the table grows by 1."""
    say("embed_grad: differences")
    rng = np.random.default_rng(10)
    w, _, _ = rand(rng, 6, 21, "f32")
    v = torch.from_numpy(ids_of(rng, 40, 8)).to(DEV)
    c, _, _ = rand(rng, 40, 21, "f32")
    d = etc.Dropout(0.3, 99, call=2)
    dt = torch.empty(6, 21, device=DEV)
    ws, _ = workspace(etc.etc_embed_grad_bytes(40, 6, 21))
    etc.etc_embed_grad(v, c, dt, ws, row0=1, scale=2.5, dropout=d)
    base = torch.empty(40, 21, device=DEV)
    etc.etc_embed(v, w, base, row0=1, scale=2.5, dropout=d)
    for r in range(6):
        for j in range(0, 21, 4):
            w2 = w.clone()
            w2[r, j] += 1.0
            out = torch.empty(40, 21, device=DEV)
            etc.etc_embed(v, w2, out, row0=1, scale=2.5, dropout=d)
            change = ((out - base).double() * c.double()).sum()
            # both outputs and w + 1 are rounded to 32 bits: 2.5 * 1.43 * (|w| + 1) * 3 u per token
            bound = 40 * 2.5 * 1.43 * 6.0 * 3 * op_ref.U * float(c.abs().max()) * 2
            assert abs(float(change) - float(dt[r, j])) <= bound, (r, j)


# ---------------------------------------------------------------------------
# dropout

DROPOUT = [
    # rows, cols, p, dtype, bias, residual, more, shift
    (1, 8, 0.1, "bf16", True, True, 0, 0),
    (1, 1, 0.5, "f32", True, True, 0, 0),
    (0, 16, 0.1, "bf16", True, True, 0, 0),
    (5, 0, 0.1, "f32", False, False, 0, 0),
    (128, 256, 0.1, "bf16", True, True, 0, 0),
    (37, 681, 0.25, "bf16", True, True, 3, 1),
    (37, 597, 0.25, "f32", True, False, 1, 3),
    (130, 63, 0.1, "f32", False, True, 0, 0),
    (3, 5001, 0.9, "bf16", True, True, 0, 5),
    (301, 17, 0.0, "bf16", True, True, 0, 0),
    (11, 2048, 1.0, "bf16", True, True, 0, 0),
    (11, 2048, 1.0 / 65536, "f32", False, False, 0, 0),
    (2100, 9, 0.4, "bf16", True, False, 2, 0),
    (70, 4104, 0.1, "f32", True, True, 0, 0),
]


@pytest.mark.parametrize("case", DROPOUT, ids=lambda c: "-".join(map(str, c)))
def test_dropout(case):
    rows, cols, p, dtype, bias, residual, more, shift = case
    say("dropout", case)
    rng = np.random.default_rng([rows, cols, 3])
    x, xn, _ = rand(rng, rows, cols, dtype, more=more, shift=shift)
    b, bn, _ = rand(rng, 1, cols, dtype, shift=shift)
    r, rn, _ = rand(rng, rows, cols, dtype, more=2 * more)
    o, full = blank(rows, cols, dtype, more=more, shift=shift)
    d = (p, (1 << 64) - 3, 7, (1 << 32) - 2)  # rows on both sides of 2^32
    etc.etc_dropout(x, o, etc.Dropout(*d), bias=b[0] if bias else None, residual=r if residual else None)
    torch.cuda.synchronize()
    close(o, op_ref.dropout(xn, bn[0] if bias else None, rn if residual else None, d), case)
    assert untouched(full, o)


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("case", DROPOUT + [(5000, 40, 0.1, "f32", True, False, 0, 0),
                                            (9001, 264, 0.1, "bf16", True, False, 0, 0),
                                            (70, 20000, 0.1, "bf16", True, False, 0, 0),
                                            (9, 1200003, 0.1, "f32", True, False, 0, 0),
                                            # on both sides of the last sizes of one launch
                                            (1024, 75, 0.1, "bf16", True, False, 5, 1),
                                            (1025, 75, 0.1, "bf16", True, False, 5, 1),
                                            (1024, 512, 0.25, "f32", True, False, 0, 0),
                                            (256, 8189, 0.1, "f32", True, False, 3, 0),
                                            (1024, 2051, 0.1, "f32", True, False, 0, 0),
                                            (3, 2796208, 0.1, "f32", True, False, 0, 0)]
                         # every kernel: types, whole blocks or not, dropout or not, few rows or many
                         + [(rows, cols, p, dtype, True, False, 1, 1) for rows in (40, 1100) for cols in (64, 63)
                            for p in (0.0, 0.1) for dtype in ("bf16", "f32")],
                         ids=lambda c: "-".join(map(str, c)))
def test_dropout_grad(case, accumulate):
    rows, cols, p, dtype, bias, _, more, shift = case
    say("dropout_grad", case, accumulate)
    rng = np.random.default_rng([rows, cols, 4])
    g, gn, _ = rand(rng, rows, cols, dtype, more=more, shift=shift)
    dx, full = blank(rows, cols, dtype, more=more, shift=shift)
    db, before, db_full = rand(rng, 1, cols, "f32", shift=shift)
    d = (p, 12345678901234567, 1, (1 << 32) - 2)
    ws, end = workspace(etc.etc_dropout_grad_bytes(rows, cols))
    etc.etc_dropout_grad(g, dx, etc.Dropout(*d), dbias=db[0] if bias else None, workspace=ws if bias else None,
                         accumulate=accumulate)
    torch.cuda.synchronize()
    want = op_ref.dropout_grad(gn, before[0] if bias else None, d, accumulate)
    close(dx, want[0] if bias else want, case)
    if bias:
        close(db[0], want[1], case)
    else:
        assert np.array_equal(db.cpu().numpy(), before)
    assert untouched(full, dx) and untouched(db_full, db) and bool((end == 0xEE).all())


def test_mask_is_a_function_of_place():
    """Kept elements are those of the definition, and a part of a batch has the
    mask that it has in the whole: by rows, in place, in both directions."""
    say("dropout: mask")
    rows, cols, p, seed = 300, 203, 0.37, 42
    kept, s = op_ref.mask(rows, cols, p, seed, call=9, row0=1000)
    one = torch.ones(rows, cols, device=DEV)
    whole = torch.empty_like(one)
    etc.etc_dropout(one, whole, etc.Dropout(p, seed, call=9, row0=1000))
    assert np.array_equal(whole.cpu().numpy() != 0, kept)
    assert abs(kept.mean() - (1 - op_ref.limit(p) / 65536)) < 5 * np.sqrt(0.25 / kept.size)
    for at, n in ((0, 1), (17, 100), (299, 1)):
        part = one[at:at + n].clone()
        etc.etc_dropout(part, part, etc.Dropout(p, seed, call=9, row0=1000 + at))
        assert torch.equal(part, whole[at:at + n])
        etc.etc_dropout_grad(one[at:at + n], part, etc.Dropout(p, seed, call=9, row0=1000 + at))
        assert torch.equal(part, whole[at:at + n])
    for other in (dict(seed=43, call=9), dict(seed=42, call=8)):
        x = torch.empty_like(one)
        etc.etc_dropout(one, x, etc.Dropout(p, other["seed"], call=other["call"], row0=1000))
        assert 0.3 < float(((x != 0) != (whole != 0)).float().mean()) < 0.6


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_dropped_values_do_not_count(dtype):
    """NaN and infinities in dropped places leave no trace in any output;
    in kept places they stay."""
    say("dropout: NaN in dropped places", dtype)
    rows, cols, d = 70, 90, (0.5, 3, 0, 0)
    kept, _ = op_ref.mask(rows, cols, *d)
    rng = np.random.default_rng(12)
    x, xn, _ = rand(rng, rows, cols, dtype)
    clean, dirty = torch.empty_like(x), torch.empty_like(x)
    bad = torch.tensor([float("nan"), float("inf"), float("-inf")], device=DEV).to(DT[dtype])
    filled = torch.where(torch.from_numpy(kept).to(DEV), x, bad[torch.arange(cols, device=DEV) % 3])
    drop = etc.Dropout(*d)
    r, _, _ = rand(rng, rows, cols, dtype)
    etc.etc_dropout(x, clean, drop, residual=r)
    etc.etc_dropout(filled, dirty, drop, residual=r)
    assert torch.equal(clean, dirty)
    out = [[torch.empty_like(x), torch.zeros(cols, device=DEV)] for _ in range(2)]
    ws, _ = workspace(etc.etc_dropout_grad_bytes(rows, cols))
    tab = [torch.empty(9, cols, device=DEV) for _ in range(2)]
    ids = torch.from_numpy(ids_of(rng, rows, 9)).to(DEV)
    ws2, _ = workspace(etc.etc_embed_grad_bytes(rows, 9, cols))
    for k, g in enumerate((x, filled)):
        etc.etc_dropout_grad(g, out[k][0], drop, dbias=out[k][1], workspace=ws)
        etc.etc_embed_grad(ids, g, tab[k], ws2, dropout=drop)
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and torch.equal(*tab)
    i, j = np.argwhere(kept)[5]
    x[i, j] = float("nan")
    etc.etc_dropout(x, dirty, drop)
    assert int(torch.isnan(dirty).sum()) == 1 and bool(torch.isnan(dirty[i, j]))


def test_outside_tokens_do_not_count():
    """A gradient row of NaN under an id outside the table changes nothing."""
    say("embed_grad: NaN under padding")
    rng = np.random.default_rng(13)
    v = ids_of(rng, 300, 20)
    v[::5] = -1
    g, _, _ = rand(rng, 300, 50, "bf16")
    ws, _ = workspace(etc.etc_embed_grad_bytes(300, 20, 50))
    got = []
    for fill in (0.0, float("nan")):
        g[::5] = fill
        dt = torch.empty(20, 50, device=DEV)
        etc.etc_embed_grad(torch.from_numpy(v).to(DEV), g, dt, ws)
        got.append(dt)
    assert torch.equal(*got) and not bool(torch.isnan(got[0]).any())


def test_in_place_and_repeated_rows():
    """out over x or over the residual, and inputs whose rows repeat (stride 0)."""
    say("dropout: in place, repeated rows")
    rng = np.random.default_rng(14)
    x, xn, _ = rand(rng, 60, 100, "bf16")
    r, rn, _ = rand(rng, 60, 100, "bf16")
    d = (0.2, 8, 1, 0)
    want = op_ref.dropout(xn, None, rn, d)
    a, b = x.clone(), r.clone()
    etc.etc_dropout(a, a, etc.Dropout(*d), residual=r)
    etc.etc_dropout(x, b, etc.Dropout(*d), residual=b)
    close(a, want, "over x")
    assert torch.equal(a, b)
    g = torch.tensor([0.5], device=DEV).to(torch.bfloat16)[None].expand(60, 1).expand(60, 100)
    one = torch.full((1, 100), 0.5, dtype=torch.bfloat16, device=DEV).expand(60, 100)
    assert one.stride(0) == 0
    dx, db = torch.empty_like(x), torch.empty(100, device=DEV)
    ws, _ = workspace(etc.etc_dropout_grad_bytes(60, 100))
    etc.etc_dropout_grad(one, dx, etc.Dropout(*d), dbias=db, workspace=ws)
    w0, w1 = op_ref.dropout_grad(np.full((60, 100), 0.5, np.float32), np.zeros(100), d, False)
    close(dx, w0, "repeated rows")
    close(db, w1, "repeated rows")
    with pytest.raises(ValueError):  # columns that are not contiguous
        etc.etc_dropout_grad(g, dx, etc.Dropout(*d))


def test_three_dimensions():
    say("three dimensions")
    rng = np.random.default_rng(15)
    w, _, _ = rand(rng, 30, 48, "bf16")
    v = torch.from_numpy(ids_of(rng, 24, 30)).to(DEV).view(4, 6)
    o3, o2 = torch.empty(4, 6, 48, dtype=torch.bfloat16, device=DEV), torch.empty(24, 48, dtype=torch.bfloat16, device=DEV)
    etc.etc_embed(v, w, o3, dropout=etc.Dropout(0.1, 1))
    etc.etc_embed(v.view(-1), w, o2, dropout=etc.Dropout(0.1, 1))
    assert torch.equal(o3.view(24, 48), o2)


# ---------------------------------------------------------------------------
# Adam

ADAM = [
    # count, first, step, weight decay, scale, zeros
    (1, 0, 1, 0.0, None, False),
    (1, 3, 1, 0.1, 0.5, False),
    (0, 5, 1, 0.1, 0.5, False),
    (7, 0, 2, 0.01, None, False),
    (128, 0, 10, 0.01, 0.25, False),
    (1000, 129, 1000, 0.0, None, False),
    (1021, 5, 100000, 0.1, 2.0, False),
    (70001, 2, 3, 0.01, None, False),
    (4096, 0, 1, 0.0, None, True),
    # a launch that reserves LDS
    (3000003, 5, 7, 0.01, 0.5, False),
]


def states(rng, n, zeros=False):
    w = rng.standard_normal(n).astype(np.float32) * 0.02
    m = rng.standard_normal(n).astype(np.float32) * 1e-3
    v = (rng.standard_normal(n).astype(np.float32) * 1e-3) ** 2
    g = rng.standard_normal(n).astype(np.float32) * 1e-3
    if zeros:  # a state that has not moved yet, and gradients of nothing
        m[:] = 0
        v[:] = 0
        g[::3] = 0
    return w, m, v, g


@pytest.mark.parametrize("case", ADAM, ids=lambda c: "-".join(map(str, c)))
def test_adam(case):
    count, first, step, decay, scale, zeros = case
    say("adam", case)
    rng = np.random.default_rng([count, first, step])
    n = first + count + 37
    w, m, v, g = states(rng, n, zeros)
    p0 = torch.from_numpy(w).to(torch.bfloat16)
    ar = [p0.to(DEV)] + [torch.from_numpy(x).to(DEV) for x in (w, m, v)]
    kw = dict(lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=decay)
    s = None if scale is None else torch.tensor([scale], device=DEV)
    gd = torch.from_numpy(g).to(DEV)
    etc.etc_adam(ar, gd, step=step, first=first, count=count, grad_scale=s, **kw)
    torch.cuda.synchronize()
    a, b = first, first + count
    want = op_ref.adam(w[a:b], m[a:b], v[a:b], g[a:b], step, scale=scale or 1.0, **kw)
    for x, name, old in zip(ar, ("param", "master", "m", "v"), (p0.float().numpy(), w, m, v)):
        close(x[a:b], want[name], (case, name))
        got = x.float().cpu().numpy()
        assert np.array_equal(got[:a], old[:a]) and np.array_equal(got[b:], old[b:]), (case, name)
    assert torch.equal(ar[0][a:b], ar[1][a:b].to(torch.bfloat16))  # the parameter is the rounded master
    assert np.array_equal(gd.cpu().numpy(), g)


def test_adam_whole_arenas_as_bytes():
    """Arenas as the migration calls take them (bytes), the whole of them by
    default; two steps equal two steps of the reference."""
    say("adam: byte arenas")
    rng = np.random.default_rng(16)
    w, m, v, g = states(rng, 2176)
    ar = [torch.from_numpy(w).to(torch.bfloat16).to(DEV).view(torch.uint8)] + \
        [torch.from_numpy(x).to(DEV).view(torch.uint8) for x in (w, m, v)]
    kw = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    etc.etc_adam(ar, torch.from_numpy(g).to(DEV).view(torch.uint8), step=1, **kw)
    want = op_ref.adam(w, m, v, g, 1, **kw)
    for k, name in ((1, "master"), (2, "m"), (3, "v")):
        close(ar[k].view(torch.float32), want[name], name)
    close(ar[0].view(torch.bfloat16), want["param"], "param")


# ---------------------------------------------------------------------------
# offsets, streams, graphs

def test_offsets_past_32_bits():
    """Rows 65536 elements apart, so the last ones lie past 2^32 elements; a
    range of the arenas that begins there."""
    say("offsets past 32 bits")
    rng = np.random.default_rng(17)
    rows, cols, ld = 66000, 40, 65536
    full = torch.empty((rows - 1) * ld + cols, dtype=torch.bfloat16, device=DEV)
    far = torch.as_strided(full, (rows, cols), (ld, 1))
    table, tn, _ = rand(rng, 8, cols, "bf16")
    far[-8:] = table
    v = np.array([rows - 8 + k for k in (0, 7, 3, 3, 5)])
    o, _ = blank(5, cols, "bf16")
    etc.etc_embed(torch.from_numpy(v).to(DEV), far, o)
    close(o, op_ref.embed(v - (rows - 8), tn), "table")
    # as x and out of a dropout, in place; the last rows are compared
    d = (0.25, 6, 0, 0)
    etc.etc_dropout(far, far, etc.Dropout(*d))
    kept = (d[0], d[1], d[2], rows - 8)
    close(far[-8:], op_ref.dropout(tn, None, None, kept), "dropout")
    far[-8:] = table
    # as the gradient of a lookup: only the last rows belong to the table
    ids = torch.full((rows,), -1, device=DEV)
    ids[-8:] = torch.arange(8, device=DEV) % 3
    dt = torch.empty(3, cols, device=DEV)
    ws, _ = workspace(etc.etc_embed_grad_bytes(rows, 3, cols))
    etc.etc_embed_grad(ids, far, dt, ws)
    close(dt, op_ref.embed_grad(np.arange(8) % 3, tn, np.zeros((3, cols))), "grad")
    del full, far
    torch.cuda.empty_cache()
    first, n = (1 << 32) + 3, 1000
    w, m, v, g = states(rng, n)
    ar = [torch.empty(first + n, dtype=t, device=DEV) for t in (torch.bfloat16,) + (torch.float32,) * 4]
    for x, y in zip(ar[1:], (w, m, v, g)):
        x[first:] = torch.from_numpy(y).to(DEV)
    kw = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
    etc.etc_adam(ar[:4], ar[4], step=2, first=first, **kw)
    want = op_ref.adam(w, m, v, g, 2, **kw)
    for x, name in zip(ar, ("param", "master", "m", "v")):
        close(x[first:], want[name], name)


def _step(rng):
    """One call of each operator on fixed buffers, and the outputs."""
    t, c = 300, 136
    w, _, _ = rand(rng, 40, c, "bf16")
    v = torch.from_numpy(ids_of(rng, t, 40)).to(DEV)
    d = etc.Dropout(0.1, 21)
    x, y, dx = (torch.empty(t, c, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    bias = w[0].clone()
    db, dt = torch.empty(c, device=DEV), torch.empty(40, c, device=DEV)
    ws1, _ = workspace(etc.etc_embed_grad_bytes(t, 40, c))
    ws2, _ = workspace(etc.etc_dropout_grad_bytes(t, c))
    ar = [w.clone().view(-1), w.float().view(-1), torch.empty(40 * c, device=DEV), torch.empty(40 * c, device=DEV)]

    def clear():
        for z in (x, y, dx, db, dt):
            z.fill_(float("nan"))
        ar[1].copy_(w.float().view(-1))
        ar[2].zero_()
        ar[3].zero_()

    def call(stream=None):
        etc.etc_embed(v, w, x, dropout=d, stream=stream)
        etc.etc_dropout(x, y, d, bias=bias, residual=x, stream=stream)
        etc.etc_dropout_grad(y, dx, d, dbias=db, workspace=ws2, stream=stream)
        etc.etc_embed_grad(v, dx, dt, ws1, dropout=d, stream=stream)
        etc.etc_adam(ar, dt.view(-1), step=1, lr=1e-3, stream=stream)

    return clear, call, [x, y, dx, db, dt] + ar


def test_other_streams():
    say("another stream")
    clear, call, out = _step(np.random.default_rng(18))
    clear()
    call()
    torch.cuda.synchronize()
    want = [z.clone() for z in out]
    s = torch.cuda.Stream()
    for given in (s, None):
        clear()
        torch.cuda.synchronize()
        if given is None:
            with torch.cuda.stream(s):
                call()
        else:
            call(given)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_in_a_graph():
    """No call allocates or synchronizes: a whole step is captured and replayed,
    with eager work and synchronizations between the replays."""
    say("a captured step")
    clear, call, out = _step(np.random.default_rng(19))
    clear()
    call()
    torch.cuda.synchronize()
    want = [z.clone() for z in out]
    g = torch.cuda.CUDAGraph()
    clear()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call()
    for replay in range(4):
        clear()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), replay
        clear()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), replay
    del g


def test_refusals_of_the_binding():
    """Tensors of other types, places and layouts, and short buffers, are refused before anything runs."""
    say("refusals")
    w = torch.zeros(4, 16, dtype=torch.bfloat16, device=DEV)
    ids = torch.zeros(3, dtype=torch.int64, device=DEV)
    out = torch.zeros(3, 16, dtype=torch.bfloat16, device=DEV)
    dt = torch.zeros(4, 16, device=DEV)
    ws = torch.zeros(etc.etc_embed_grad_bytes(3, 4, 16), dtype=torch.uint8, device=DEV)
    wrong = [
        lambda: etc.etc_embed(ids, w.half(), out),
        lambda: etc.etc_embed(ids.float(), w, out),
        lambda: etc.etc_embed(ids.cpu(), w, out),
        lambda: etc.etc_embed(ids, w.cpu(), out),
        lambda: etc.etc_embed(ids, w, out.cpu()),
        lambda: etc.etc_embed(ids, w.t().contiguous().t(), out),
        lambda: etc.etc_embed(torch.zeros(6, dtype=torch.int64, device=DEV)[::2], w, out),
        lambda: etc.etc_embed_grad(ids, out, dt, ws.cpu()),
        lambda: etc.etc_dropout(out.view(3, 4, 4).transpose(0, 1), out),
        lambda: etc.etc_adam([w, dt, dt, dt], dt[:2], step=1, lr=1e-3),
        lambda: etc.etc_adam([w, dt, dt], dt, step=1, lr=1e-3),
        lambda: etc.etc_adam([w, dt, dt, dt], dt, step=1, lr=1e-3, count=65),
        lambda: etc.etc_adam([w, dt, dt, dt], dt, step=1, lr=1e-3, grad_scale=torch.ones(1, device=DEV).double()),
    ]
    for k, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            say("not refused:", k)
    refused = [
        (lambda: etc.etc_embed(ids, w, out[:2]), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed(ids, w, out[:, :8]), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed(ids, w, out, positions=ids), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed(ids, w, out[:1].expand(3, 16)), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed_grad(ids, out, dt.bfloat16(), ws), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed_grad(ids, out, dt, ws[:-1]), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed_grad(ids, out, dt, None), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_embed_grad(ids, out, dt, torch.zeros(ws.numel() + 256, dtype=torch.uint8, device=DEV)[8:]),
         etc.ERR_ALIGN),
        (lambda: etc.etc_dropout(out, out, bias=dt[0]), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_dropout_grad(out, out, dbias=dt[0]), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_adam([w, dt, dt, dt], dt, step=0, lr=1e-3), etc.ERR_INVALID_ARG),
        (lambda: etc.etc_adam([w, dt, dt, dt], dt, step=1, lr=1e-3, beta2=1.0), etc.ERR_INVALID_ARG),
    ]
    for call, code in refused:
        with pytest.raises(etc.EtcError) as e:
            call()
        assert e.value.code == code
    torch.cuda.synchronize()
    assert not bool(dt.any()) and not bool(out.any()) and not bool(w.any())
