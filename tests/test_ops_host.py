"""The operators of a training step without a GPU: dropout's generator against
its published known answers, the helpers of the launches, the layout of the
argument structs, and the refusals of the C ABI (arguments are checked before
anything is launched)."""
import ctypes
import hashlib
import os
import subprocess

import numpy as np
import pytest

import op_ref
from paper_2607_04749_amd import etc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_04749_amd", "csrc")
SRC = os.path.join(ROOT, "tests", "opshost", "opshost.cpp")


@pytest.fixture(scope="module")
def host():
    files = [SRC] + [os.path.join(CSRC, f) for f in ("ops.hpp", "philox.hpp")] + [os.path.join(ROOT, "include", "etc.h")]
    h = hashlib.sha256(b"".join(open(f, "rb").read() for f in files)).hexdigest()[:16]
    out = os.path.join(ROOT, "_build", "opshost", h)
    if not os.path.exists(out):
        os.makedirs(os.path.dirname(out), exist_ok=True)
        part = f"{out}.{os.getpid()}"  # several test processes may build it at once
        r = subprocess.run(["hipcc", "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang",
                            "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"),
                            "-I", CSRC, SRC, "-o", part], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        os.replace(part, out)

    def run(*args):
        r = subprocess.run([out, *map(str, args)], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return r.stdout
    return run


# counter, key, words: the answers published with the generator
KNOWN = [((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
         ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
         ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
          (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]


def test_generator(host):
    rng = np.random.default_rng(1)
    for counter, key, words in KNOWN:
        assert tuple(int(x) for x in op_ref.philox(counter, key)) == words
    for counter, key in [(c, k) for c, k, _ in KNOWN] + \
            [(rng.integers(0, 1 << 32, 4), rng.integers(0, 1 << 32, 2)) for _ in range(20)]:
        got = host("philox", *("%x" % int(x) for x in (*counter, *key))).split()
        assert [int(x, 16) for x in got] == [int(x) for x in op_ref.philox(counter, key)]


def test_kept_share():
    """The share kept is that of the limit, over rows, columns and the places in a block of eight."""
    for p in (0.1, 0.5, 0.9):
        kept, scale = op_ref.mask(2000, 256, p, 7, call=1)
        q = 1 - op_ref.limit(p) / 65536
        assert abs(scale * q - 1) < 1e-12
        assert abs(kept.mean() - q) < 5 * np.sqrt(q * (1 - q) / kept.size)
        by_place = kept.reshape(2000, 32, 8).mean((0, 1))
        assert np.abs(by_place - q).max() < 5 * np.sqrt(q * (1 - q) / 64000)
        left, right = kept[:, :-1] - q, kept[:, 1:] - q
        assert abs((left * right).mean()) < 5 * q * (1 - q) / np.sqrt(left.size)


def test_division(host):
    assert host("divide").strip() == "0"


@pytest.mark.parametrize("rows,cols", [(1, 1), (1000, 8), (1, (1 << 31) - 1), ((1 << 31) - 1, 8), ((1 << 31) - 1, 4097),
                                       (3, (1 << 31) - 1)])
@pytest.mark.parametrize("block,per", ((8, 1), (8, 2), (4, 1)))
def test_launches_cover_the_rows(host, rows, cols, block, per):
    nb, at = -(-cols // block), 0
    for line in host("runs", rows, cols, block, per).splitlines():
        first, n, run, c, d = map(int, line.split())
        assert first == at and c == cols and d == nb
        assert n == -(-run // per) * nb and 0 < n < 2 ** 31
        at += run
        # only the last run ends inside a lane's rows or leaves room for more
        assert at == rows or (run % per == 0 and n + nb >= 2 ** 31)
    assert at == rows


def test_layout(host):
    got = dict(line.split() for line in host("layout").splitlines())
    got = {k: int(v) for k, v in got.items()}
    size = lambda f: __import__("struct").calcsize("@" + f)  # noqa: E731
    m, i, d = etc._MATRIX, etc._IDS, etc._DROP
    assert (size(m), size(i), size(d)) == (got["etc_matrix"], got["etc_ids"], got["etc_dropout_desc"])
    for name, packed in (("etc_embed_args", etc._EMBED), ("etc_embed_grad_args", etc._EMBED_GRAD),
                         ("etc_dropout_args", etc._DROPOUT), ("etc_dropout_grad_args", etc._DROPOUT_GRAD),
                         ("etc_adam_args", etc._ADAM)):
        assert packed.size == got[name], name
    assert got["etc_embed_args.table"] == size(2 * i) and got["etc_embed_args.drop"] == size(2 * i + 3 * m)
    assert got["etc_embed_args.row0"] == size(2 * i + 3 * m + d)
    assert got["etc_embed_grad_args.workspace"] == size(i + 2 * m + d + "qd")
    assert got["etc_embed_grad_args.accumulate"] == size(i + 2 * m + d + "qdPQ")
    assert got["etc_dropout_args.drop"] == size(4 * m) and got["etc_dropout_grad_args.drop"] == size(3 * m)
    assert got["etc_adam_args.first"] == size("6P") and got["etc_adam_args.step"] == size("6PQQ5d")


# ---- refusals: the pointers below are never followed ----

PTR = 1 << 20


def mat(rows, cols, dtype=etc.DTYPE_BF16, ptr=PTR, ld=None, reserved=0):
    return (ptr, rows, cols, cols if ld is None else ld, dtype, reserved)


def ids(n, ptr=PTR, dtype=etc.IDS_I64, reserved=0):
    return (ptr, n, dtype, reserved)


def drop(p=0.1, row0=0, reserved=0):
    return (1, row0, p, 0, reserved)


NONE, NO_IDS = etc._NO_MATRIX, etc._NO_IDS
NAN = float("nan")


def embed(tokens=ids(3), positions=NO_IDS, table=mat(9, 16), pos=NONE, out=mat(3, 16), d=drop(), scale=1.0):
    return etc.lib().etc_embed(etc._EMBED.pack(*tokens, *positions, *table, *pos, *out, *d, 0, scale), None)


def embed_grad(tokens=ids(3), grad=mat(3, 16), dtable=mat(9, 16, etc.DTYPE_F32), d=drop(), scale=1.0, ws=PTR,
               nbytes=1 << 30, accumulate=0, reserved=0):
    return etc.lib().etc_embed_grad(
        etc._EMBED_GRAD.pack(*tokens, *grad, *dtable, *d, 0, scale, ws, nbytes, accumulate, reserved), None)


def dropout(x=mat(3, 16), bias=NONE, residual=NONE, out=mat(3, 16), d=drop()):
    return etc.lib().etc_dropout(etc._DROPOUT.pack(*x, *bias, *residual, *out, *d), None)


def dropout_grad(grad=mat(3, 16), dx=mat(3, 16), dbias=NONE, d=drop(), ws=PTR, nbytes=1 << 30, accumulate=0,
                 reserved=0):
    return etc.lib().etc_dropout_grad(
        etc._DROPOUT_GRAD.pack(*grad, *dx, *dbias, *d, ws, nbytes, accumulate, reserved), None)


def adam(arenas=(PTR,) * 4, grad=PTR, scale=0, first=0, count=8, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, step=1):
    return etc.lib().etc_adam(etc._ADAM.pack(*arenas, grad, scale, first, count, lr, b1, b2, eps, wd, step), None)


F32 = etc.DTYPE_F32
INVALID, ALIGN, UNSUPPORTED, OK = etc.ERR_INVALID_ARG, etc.ERR_ALIGN, etc.ERR_UNSUPPORTED, etc.OK
REFUSED = [
    (lambda: embed(tokens=ids(3, ptr=0)), INVALID), (lambda: embed(tokens=ids(3, dtype=2)), INVALID),
    (lambda: embed(tokens=ids(-1)), INVALID), (lambda: embed(tokens=ids(3, reserved=1)), INVALID),
    (lambda: embed(tokens=ids(1 << 31), out=mat(1 << 31, 16)), UNSUPPORTED),
    (lambda: embed(tokens=ids(3, ptr=PTR + 4)), ALIGN),
    (lambda: embed(table=mat(9, 16, ptr=0)), INVALID), (lambda: embed(table=mat(9, 16, ptr=PTR + 1)), ALIGN),
    (lambda: embed(table=mat(9, 16, dtype=7)), INVALID), (lambda: embed(table=mat(9, 15)), INVALID),
    (lambda: embed(table=mat(9, 16, ld=-1)), INVALID), (lambda: embed(table=mat(9, 16, ld=1 << 60)), INVALID),
    (lambda: embed(table=mat(1 << 31, 16)), UNSUPPORTED), (lambda: embed(table=mat(9, 16, reserved=1)), INVALID),
    (lambda: embed(out=mat(3, 16, ld=15)), INVALID), (lambda: embed(out=mat(2, 16)), INVALID),
    (lambda: embed(out=mat(3, 16, ptr=0)), INVALID), (lambda: embed(out=mat(3, 16, F32, ptr=PTR + 2)), ALIGN),
    (lambda: embed(positions=ids(3)), INVALID), (lambda: embed(pos=mat(4, 16)), INVALID),
    (lambda: embed(positions=ids(2), pos=mat(4, 16)), INVALID),
    (lambda: embed(positions=ids(3), pos=mat(4, 8)), INVALID),
    (lambda: embed(positions=ids(3), pos=mat(4, 16, F32)), INVALID),
    (lambda: embed(scale=NAN), INVALID), (lambda: embed(scale=float("inf")), INVALID),
    (lambda: embed(d=drop(p=-0.1)), INVALID), (lambda: embed(d=drop(p=1.1)), INVALID),
    (lambda: embed(d=drop(p=NAN)), INVALID), (lambda: embed(d=drop(row0=-1)), INVALID),
    (lambda: embed(d=drop(row0=(1 << 63) - 2)), INVALID), (lambda: embed(d=drop(reserved=1)), INVALID),
    (lambda: embed_grad(tokens=ids(4)), INVALID), (lambda: embed_grad(grad=mat(3, 8)), INVALID),
    (lambda: embed_grad(dtable=mat(9, 16)), INVALID), (lambda: embed_grad(dtable=mat(9, 16, F32, ld=8)), INVALID),
    (lambda: embed_grad(ws=0), INVALID), (lambda: embed_grad(ws=PTR + 128), ALIGN),
    (lambda: embed_grad(nbytes=8), INVALID), (lambda: embed_grad(reserved=1), INVALID),
    (lambda: embed_grad(tokens=ids((1 << 31) - 1), grad=mat((1 << 31) - 1, (1 << 31) - 1, ld=0),
                        dtable=mat(1, (1 << 31) - 1, F32)), UNSUPPORTED),
    (lambda: embed_grad(tokens=ids((1 << 27) + 1), grad=mat((1 << 27) + 1, 16)), UNSUPPORTED),
    (lambda: embed_grad(scale=NAN), INVALID), (lambda: embed_grad(d=drop(p=2.0)), INVALID),
    (lambda: dropout(out=mat(3, 16, F32)), INVALID), (lambda: dropout(out=mat(3, 17)), INVALID),
    (lambda: dropout(bias=mat(2, 16)), INVALID), (lambda: dropout(bias=mat(1, 8)), INVALID),
    (lambda: dropout(bias=mat(1, 16, F32)), INVALID), (lambda: dropout(residual=mat(3, 16, F32)), INVALID),
    (lambda: dropout(residual=mat(4, 16)), INVALID), (lambda: dropout(x=mat(3, -1)), INVALID),
    (lambda: dropout(d=drop(p=NAN)), INVALID),
    (lambda: dropout_grad(dx=mat(3, 16, F32)), INVALID), (lambda: dropout_grad(dbias=mat(1, 16)), INVALID),
    (lambda: dropout_grad(dbias=mat(1, 15, F32)), INVALID), (lambda: dropout_grad(dbias=mat(1, 16, F32), ws=0), INVALID),
    (lambda: dropout_grad(dbias=mat(1, 16, F32), ws=PTR + 4), ALIGN),
    (lambda: dropout_grad(dbias=mat(1, 16, F32), nbytes=4), INVALID), (lambda: dropout_grad(reserved=1), INVALID),
    (lambda: adam(arenas=(PTR, 0, PTR, PTR)), INVALID), (lambda: adam(arenas=(PTR, PTR, PTR + 4, PTR)), ALIGN),
    (lambda: adam(grad=0), INVALID), (lambda: adam(grad=PTR + 8), ALIGN), (lambda: adam(scale=PTR + 2), ALIGN),
    (lambda: adam(step=0), INVALID), (lambda: adam(b1=1.0), INVALID), (lambda: adam(b2=-0.1), INVALID),
    (lambda: adam(b1=NAN), INVALID), (lambda: adam(eps=-1.0), INVALID), (lambda: adam(lr=NAN), INVALID),
    (lambda: adam(wd=float("inf")), INVALID), (lambda: adam(count=1 << 62), INVALID),
    (lambda: adam(first=1 << 62), INVALID),
]


@pytest.mark.parametrize("k", range(len(REFUSED)))
def test_refusals(k):
    call, code = REFUSED[k]
    assert call() == code, (k, etc.last_error())
    assert etc.last_error()


def test_null_arguments():
    for name in ("etc_embed", "etc_embed_grad", "etc_dropout", "etc_dropout_grad", "etc_adam"):
        assert getattr(etc.lib(), name)(None, None) == INVALID
    assert etc.lib().etc_embed_grad_workspace(1, 1, 1, None) == INVALID
    assert etc.lib().etc_dropout_grad_workspace(1, 1, None) == INVALID
    n = ctypes.c_uint64()
    assert etc.lib().etc_embed_grad_workspace(-1, 1, 1, ctypes.byref(n)) == INVALID
    assert etc.lib().etc_embed_grad_workspace(1, 1 << 31, 1, ctypes.byref(n)) == UNSUPPORTED
    assert etc.lib().etc_dropout_grad_workspace(1, -1, ctypes.byref(n)) == INVALID


def test_calls_without_work():
    """Nothing to compute: OK, with nothing launched and no pointer followed."""
    assert embed(tokens=ids(0, ptr=0), out=mat(0, 16, ptr=0)) == OK
    assert embed(table=mat(9, 0, ptr=0), out=mat(3, 0, ptr=0)) == OK
    assert embed(tokens=ids(0, ptr=0), out=mat(0, 16, ptr=0), positions=ids(0, ptr=0), pos=mat(4, 16)) == OK
    assert embed(tokens=ids(0, ptr=0), out=mat(0, 16, ptr=0), positions=ids(0, ptr=0), pos=mat(0, 16, ptr=0)) == OK
    assert embed_grad(tokens=ids(0, ptr=0), grad=mat(0, 16, ptr=0), accumulate=1) == OK
    assert embed_grad(dtable=mat(0, 16, F32, ptr=0)) == OK
    assert dropout(x=mat(0, 16, ptr=0), out=mat(0, 16, ptr=0)) == OK
    assert dropout_grad(grad=mat(0, 16, ptr=0), dx=mat(0, 16, ptr=0)) == OK
    assert dropout_grad(grad=mat(0, 16, ptr=0), dx=mat(0, 16, ptr=0), dbias=mat(1, 16, F32), accumulate=1) == OK
    assert adam(count=0) == OK


def test_workspaces_grow_with_their_sizes():
    """A workspace for larger sizes serves smaller ones."""
    sizes = (0, 1, 63, 64, 65, 1000, 4096, 8192, 8193, 30000, 65537, 1 << 20)
    for cols in (1, 8, 513, 8192):
        got = [etc.etc_embed_grad_bytes(n, 1000, cols) for n in sizes]
        assert got == sorted(got)
        got = [etc.etc_dropout_grad_bytes(n, cols) for n in sizes]
        assert got == sorted(got) and got[0] == 0
    assert etc.etc_embed_grad_bytes(8192, 50304, 2048) < 64 << 20
    rng = np.random.default_rng(2)
    for ask in (lambda n, c: etc.etc_embed_grad_bytes(n, 9, c), etc.etc_dropout_grad_bytes):
        for _ in range(2000):
            n, c = (int(np.exp(rng.random() * np.log(hi))) for hi in (1 << 20, 20000))
            more = int(np.exp(rng.random() * np.log(1 + n)))
            assert ask(n, c) <= ask(n + more, c) and ask(n, c) <= ask(n, c + 1) and ask(n, c) <= ask(n, 2 * c)


@pytest.mark.parametrize("bad", (dict(p=-0.1), dict(p=1.5), dict(p=NAN), dict(seed=-1), dict(seed=1 << 64),
                                 dict(call=1 << 32), dict(row0=-1), dict(row0=1 << 63)))
def test_dropout_object_refuses(bad):
    with pytest.raises(ValueError):
        etc.Dropout(**{**dict(p=0.1, seed=0), **bad})
