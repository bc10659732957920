"""The operators around a block's projections without a GPU: the layout of the
argument structs, the refusals of the C ABI (arguments are checked before anything
is launched), the frequencies of rotary positions, workspaces, what the binding hands
over and refuses, and the plain implementation against differences."""
import ctypes
import hashlib
import math
import os
import struct
import subprocess

import numpy as np
import pytest
import torch

import block_ref
from paper_2607_04749_amd import etc
from test_ops_host import ALIGN, F32, INVALID, NO_IDS, NONE, OK, PTR, UNSUPPORTED, ids, mat

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "blockhost", "layout.cpp")
NAN, INF = float("nan"), float("inf")


def test_layout():
    files = [SRC, os.path.join(ROOT, "include", "etc.h")]
    h = hashlib.sha256(b"".join(open(f, "rb").read() for f in files)).hexdigest()[:16]
    out = os.path.join(ROOT, "_build", "blockhost", h)
    if not os.path.exists(out):
        os.makedirs(os.path.dirname(out), exist_ok=True)
        part = f"{out}.{os.getpid()}"  # several test processes may build it at once
        subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), SRC, "-o", part], check=True)
        os.replace(part, out)
    got = {k: int(v) for k, v in (line.split() for line in
                                  subprocess.run([out], capture_output=True, text=True, check=True).stdout.splitlines())}
    size = lambda f: struct.calcsize("@" + f)  # noqa: E731
    m, m8, i = etc._MATRIX, etc._MATRIX8, etc._IDS
    want = {
        "etc_matrix8": size(m8), "etc_matrix8.scale": size("P"), "etc_matrix8.rows": size("PP"),
        "etc_matrix8.scale_ld": size("PPqqq"), "etc_matrix8.group": size("PPqqqqi"),
        "etc_norm_args": etc._NORM.size, "etc_norm_args.weight": size(2 * m), "etc_norm_args.out8": size(5 * m),
        "etc_norm_args.rstd": size(5 * m + m8), "etc_norm_args.eps": size(5 * m + m8 + "P"),
        "etc_norm_grad_args": etc._NORM_GRAD.size, "etc_norm_grad_args.x8": size(2 * m),
        "etc_norm_grad_args.dweight": size(5 * m + m8), "etc_norm_grad_args.rstd": size(6 * m + m8),
        "etc_norm_grad_args.workspace_bytes": size(6 * m + m8 + "PP"), "etc_norm_grad_args.accumulate": size(6 * m + m8 + "PPQ"),
        "etc_store8_args": etc._STORE8.size, "etc_store8_args.col_scale": size(m), "etc_store8_args.out": size(m + "P"),
        "etc_load8_args": etc._LOAD8.size, "etc_load8_args.out": size(m8),
        "etc_matmul8_args": etc._MATMUL8.size, "etc_matmul8_args.w": size(m8), "etc_matmul8_args.bias": size(2 * m8),
        "etc_matmul8_args.out": size(2 * m8 + m),
        "etc_rotary_desc": ctypes.sizeof(etc.RotaryDesc), "etc_rotary_desc.scale": etc.RotaryDesc.scale.offset,
        "etc_rotary_desc.pairs": etc.RotaryDesc.pairs.offset, "etc_rotary_desc.layout": etc.RotaryDesc.layout.offset,
        "etc_rotary_args": etc._ROTARY.size, "etc_rotary_args.positions": size(2 * m), "etc_rotary_args.rotary": size(2 * m + i),
        "etc_rotary_args.head_dim": size(2 * m + i + "P"), "etc_rotary_args.backward": size(2 * m + i + "Pi"),
    }
    assert got == want


# ---- refusals: the pointers below are never followed ----

I8, E4M3 = etc.DTYPE_I8, etc.DTYPE_E4M3
NO8 = etc._NO_MATRIX8


def mat8(rows, cols, dtype=I8, group=0, ptr=PTR, scale=PTR, ld=None, sld=None):
    n = -(-cols // group) if group > 0 else 1
    return (ptr, scale, rows, cols, cols if ld is None else ld, n if sld is None else sld, dtype, group)


def norm(x=mat(3, 16), residual=NONE, weight=mat(1, 16), sum=NONE, out=mat(3, 16), out8=NO8, rstd=0, eps=1e-6):
    return etc.lib().etc_norm(etc._NORM.pack(*x, *residual, *weight, *sum, *out, *out8, rstd, eps), None)


def norm_grad(grad=mat(3, 16), x=mat(3, 16), x8=NO8, weight=mat(1, 16), dsum=NONE, dx=mat(3, 16), dweight=NONE, rstd=PTR,
              ws=PTR, nbytes=1 << 30, accumulate=0, reserved=0):
    return etc.lib().etc_norm_grad(etc._NORM_GRAD.pack(*grad, *x, *x8, *weight, *dsum, *dx, *dweight, rstd, ws, nbytes,
                                                       accumulate, reserved), None)


def store8(x=mat(3, 16), col_scale=0, out=mat8(3, 16)):
    return etc.lib().etc_store8(etc._STORE8.pack(*x, col_scale, *out), None)


def load8(x=mat8(3, 16), out=mat(3, 16)):
    return etc.lib().etc_load8(etc._LOAD8.pack(*x, *out), None)


def matmul8(x=mat8(3, 16), w=mat8(5, 16), bias=NONE, out=mat(3, 5)):
    return etc.lib().etc_matmul8(etc._MATMUL8.pack(*x, *w, *bias, *out), None)


def desc(pairs=4, layout=0, scale=1.0, freq=1.0):
    d = etc.RotaryDesc()
    for j in range(etc.ROTARY_PAIRS):
        d.freq[j] = freq
    d.scale, d.pairs, d.layout = scale, pairs, layout
    return d


def rotary(x=mat(3, 16), out=mat(3, 16), positions=ids(3), d=desc(), head_dim=8, backward=0):
    at = 0 if d is None else ctypes.addressof(d)
    return etc.lib().etc_rotary(etc._ROTARY.pack(*x, *out, *positions, at, head_dim, backward), None)


BIG = (1 << 31) - 1
REFUSED = [
    (lambda: norm(x=mat(3, 16, ptr=0)), INVALID), (lambda: norm(x=mat(3, 16, ptr=PTR + 1)), ALIGN),
    (lambda: norm(x=mat(3, 16, dtype=2)), INVALID), (lambda: norm(x=mat(1 << 31, 16), out=mat(1 << 31, 16)), UNSUPPORTED),
    (lambda: norm(weight=mat(1, 15)), INVALID), (lambda: norm(weight=mat(2, 16)), INVALID),
    (lambda: norm(weight=mat(1, 16, F32)), INVALID), (lambda: norm(weight=mat(1, 16, ptr=0)), INVALID),
    (lambda: norm(residual=mat(3, 15)), INVALID), (lambda: norm(residual=mat(3, 16, F32)), INVALID),
    (lambda: norm(sum=mat(3, 16, ptr=2 * PTR, ld=15)), INVALID), (lambda: norm(sum=mat(4, 16, ptr=2 * PTR)), INVALID),
    (lambda: norm(sum=mat(3, 16, F32, ptr=2 * PTR)), INVALID), (lambda: norm(sum=mat(3, 16)), INVALID),
    (lambda: norm(out=mat(3, 16, F32)), INVALID), (lambda: norm(out=mat(3, 16, ld=8)), INVALID),
    (lambda: norm(out=NONE), INVALID), (lambda: norm(out=NONE, out8=mat8(3, 15)), INVALID),
    (lambda: norm(out8=mat8(3, 16, group=32)), INVALID), (lambda: norm(out8=mat8(3, 16, dtype=0)), INVALID),
    (lambda: norm(out8=mat8(3, 16, scale=0)), INVALID), (lambda: norm(out8=mat8(3, 16, scale=PTR + 2)), ALIGN),
    (lambda: norm(sum=mat(3, 16, ld=24)), INVALID), (lambda: norm(out=mat(3, 16, ld=24)), INVALID),
    (lambda: norm(residual=mat(3, 16, ptr=4 * PTR), sum=mat(3, 16, ptr=4 * PTR, ld=24)), INVALID),
    (lambda: norm_grad(dx=mat(3, 16, ptr=4 * PTR, ld=24), dsum=mat(3, 16, ptr=4 * PTR)), INVALID),
    (lambda: norm(out8=mat8(3, 16, ld=15)), INVALID), (lambda: norm(out8=mat8(3, 16, sld=0)), INVALID),
    (lambda: norm(rstd=PTR + 1), ALIGN), (lambda: norm(eps=0.0), INVALID), (lambda: norm(eps=-1.0), INVALID),
    (lambda: norm(eps=NAN), INVALID), (lambda: norm(eps=INF), INVALID), (lambda: norm(eps=1e39), INVALID),
    (lambda: norm(eps=1e-60), INVALID),
    (lambda: norm_grad(grad=mat(3, 16, ptr=0)), INVALID), (lambda: norm_grad(dx=mat(3, 16, F32)), INVALID),
    (lambda: norm_grad(dx=mat(3, 15)), INVALID), (lambda: norm_grad(dx=mat(3, 16, ld=3)), INVALID),
    (lambda: norm_grad(x=NONE), INVALID), (lambda: norm_grad(x=mat(3, 16, F32)), INVALID), (lambda: norm_grad(x=mat(2, 16)), INVALID),
    (lambda: norm_grad(x8=mat8(3, 16)), INVALID), (lambda: norm_grad(x=NONE, x8=mat8(3, 8)), INVALID),
    (lambda: norm_grad(x=NONE, x8=mat8(3, 16, scale=0)), INVALID), (lambda: norm_grad(x=NONE, x8=mat8(3, 16, group=16)), INVALID),
    (lambda: norm_grad(x=NONE, x8=mat8(3, 16, group=-32)), INVALID), (lambda: norm_grad(x=NONE, x8=mat8(3, 16, ld=-1)), INVALID),
    (lambda: norm_grad(x=NONE, x8=mat8(3, 16, sld=-1)), INVALID), (lambda: norm_grad(x=NONE, x8=mat8(3, 16, sld=1 << 61)), INVALID),
    (lambda: norm_grad(weight=mat(1, 16, F32)), INVALID), (lambda: norm_grad(weight=mat(3, 16)), INVALID),
    (lambda: norm_grad(dsum=mat(3, 17)), INVALID), (lambda: norm_grad(rstd=0), INVALID), (lambda: norm_grad(rstd=PTR + 2), ALIGN),
    (lambda: norm_grad(dweight=mat(1, 16)), INVALID), (lambda: norm_grad(dweight=mat(1, 15, F32)), INVALID),
    (lambda: norm_grad(dweight=mat(1, 16, F32), ws=0), INVALID), (lambda: norm_grad(dweight=mat(1, 16, F32), ws=PTR + 16), ALIGN),
    (lambda: norm_grad(dweight=mat(1, 16, F32), nbytes=16), INVALID), (lambda: norm_grad(reserved=1), INVALID),
    (lambda: store8(out=mat8(3, 17)), INVALID), (lambda: store8(out=mat8(2, 16)), INVALID), (lambda: store8(out=mat8(3, 16, ptr=0)), INVALID),
    (lambda: store8(out=mat8(3, 16, group=512)), INVALID), (lambda: store8(out=mat8(3, 16, group=1)), INVALID),
    (lambda: store8(x=mat(3, 40), out=mat8(3, 40, group=32, sld=1)), INVALID), (lambda: store8(col_scale=PTR + 1), ALIGN),
    (lambda: store8(x=mat(3, 16, dtype=3)), INVALID), (lambda: store8(out=mat8(3, 16, ld=1 << 60)), INVALID),
    (lambda: load8(x=mat8(3, 17)), INVALID), (lambda: load8(x=mat8(3, 16, scale=0)), INVALID), (lambda: load8(x=mat8(3, 16, dtype=1)), INVALID),
    (lambda: load8(out=mat(3, 16, ld=15)), INVALID), (lambda: load8(out=mat(3, 16, F32, ptr=PTR + 2)), ALIGN),
    (lambda: matmul8(x=mat8(3, 17)), INVALID), (lambda: matmul8(x=mat8(3, 16, dtype=E4M3)), INVALID),
    (lambda: matmul8(w=mat8(5, 16, dtype=E4M3)), INVALID), (lambda: matmul8(w=mat8(5, 16, group=32)), INVALID),
    (lambda: matmul8(x=mat8(3, 16, group=32)), INVALID), (lambda: matmul8(out=mat(3, 6)), INVALID), (lambda: matmul8(out=mat(4, 5)), INVALID),
    (lambda: matmul8(out=mat(3, 5, ld=4)), INVALID), (lambda: matmul8(bias=mat(1, 5, F32)), INVALID), (lambda: matmul8(bias=mat(1, 4)), INVALID),
    (lambda: matmul8(bias=mat(1, 5, ptr=PTR + 1)), ALIGN), (lambda: matmul8(x=mat8(3, 16, ptr=0)), INVALID),
    (lambda: matmul8(x=mat8(3, 131072), w=mat8(5, 131072)), UNSUPPORTED), (lambda: matmul8(x=mat8(3, 16, scale=PTR + 3)), ALIGN),
    (lambda: rotary(out=mat(3, 16, F32)), INVALID), (lambda: rotary(out=mat(3, 8)), INVALID), (lambda: rotary(x=mat(3, 16, ptr=0)), INVALID),
    (lambda: rotary(out=mat(3, 16, ld=15)), INVALID), (lambda: rotary(positions=ids(2)), INVALID), (lambda: rotary(positions=ids(3, ptr=0)), INVALID),
    (lambda: rotary(positions=ids(3, ptr=PTR + 4)), ALIGN), (lambda: rotary(positions=ids(3, dtype=5)), INVALID),
    (lambda: rotary(d=None), INVALID), (lambda: rotary(d=desc(pairs=0)), INVALID), (lambda: rotary(d=desc(pairs=129), head_dim=16), INVALID),
    (lambda: rotary(d=desc(layout=2)), INVALID), (lambda: rotary(d=desc(scale=INF)), INVALID), (lambda: rotary(d=desc(scale=1e39)), INVALID),
    (lambda: rotary(d=desc(freq=NAN)), INVALID), (lambda: rotary(d=desc(pairs=5)), INVALID), (lambda: rotary(head_dim=0), INVALID),
    (lambda: rotary(head_dim=12), INVALID), (lambda: rotary(head_dim=-8), INVALID), (lambda: rotary(x=mat(3, 16, ld=17)), INVALID),
]


@pytest.mark.parametrize("k", range(len(REFUSED)))
def test_refusals(k):
    call, code = REFUSED[k]
    assert call() == code, (k, etc.last_error())
    assert etc.last_error()


def test_null_arguments():
    for name in ("etc_norm", "etc_norm_grad", "etc_store8", "etc_load8", "etc_matmul8", "etc_rotary"):
        assert getattr(etc.lib(), name)(None, None) == INVALID
    n = ctypes.c_uint64()
    assert etc.lib().etc_norm_grad_workspace(1, 1, None) == INVALID
    assert etc.lib().etc_norm_grad_workspace(-1, 1, ctypes.byref(n)) == INVALID
    assert etc.lib().etc_norm_grad_workspace(1, 1 << 31, ctypes.byref(n)) == UNSUPPORTED
    assert etc.lib().etc_rotary_init(None, 8, 0, 1e4, 0, 1.0, 0.0, 0.0, 1.0) == INVALID


def test_calls_without_work():
    """Nothing to compute: OK, with nothing launched and no pointer followed."""
    e = mat(0, 16, ptr=0)
    assert norm(x=e, out=NONE) == OK and norm(x=mat(3, 0, ptr=0), weight=NONE, out=NONE) == OK
    assert norm_grad(grad=e, x=e, dx=e, rstd=0) == OK
    assert norm_grad(grad=e, x=e, dx=e, rstd=0, dweight=mat(1, 16, F32), accumulate=1) == OK
    none = mat(3, 0, ptr=0)
    assert norm_grad(grad=none, x=none, dx=none, weight=NONE, rstd=0) == OK
    assert store8(x=e, out=mat8(0, 16, ptr=0, scale=0)) == OK and store8(x=none, out=mat8(3, 0, ptr=0, scale=0)) == OK
    assert load8(x=mat8(0, 16, ptr=0, scale=0), out=e) == OK and load8(x=mat8(3, 0, ptr=0, scale=0), out=none) == OK
    assert matmul8(x=mat8(0, 16, ptr=0, scale=0), out=mat(0, 5, ptr=0)) == OK
    assert matmul8(w=mat8(0, 16, ptr=0, scale=0), out=mat(3, 0, ptr=0)) == OK
    assert rotary(x=e, out=e, positions=ids(0, ptr=0)) == OK and rotary(x=none, out=none) == OK


def test_workspace_grows_with_its_sizes():
    rng = np.random.default_rng(2)
    ask = etc.etc_norm_grad_bytes
    assert ask(0, 100) == 0 and ask(8192, 4096) <= 64 << 20
    for _ in range(2000):
        n, c = (int(np.exp(rng.random() * np.log(hi))) for hi in (1 << 20, 200000))
        more = int(np.exp(rng.random() * np.log(1 + n)))
        assert ask(n, c) <= ask(n + more, c) and ask(n, c) <= ask(n, c + 1) and ask(n, c) <= ask(n, 2 * c)


# ---- rotary frequencies ----

@pytest.mark.parametrize("dim", (2, 4, 52, 128, 256))
@pytest.mark.parametrize("kw", (dict(), dict(base=5e5), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                dict(scaling="parts", factor=8.0, length=4096.0, low=1.0, high=32.0),
                                dict(scaling="parts", factor=32.0, length=8192.0, low=1.0, high=4.0, base=5e5)))
def test_frequencies(dim, kw):
    if dim == 2 and kw.get("scaling") == "base":
        with pytest.raises(etc.EtcError):
            etc.Rotary(dim, **kw)
        return
    got, want = np.array(etc.Rotary(dim, **kw).freq), block_ref.frequencies(dim, **kw)
    assert got.shape == (dim // 2,) and np.allclose(got, want, rtol=1e-13, atol=0)
    if kw.get("scaling") == "base":  # the fastest pair as it was, the slowest one's divided by the factor
        plain = np.array(etc.Rotary(dim).freq)
        assert got[0] == plain[0] and math.isclose(got[-1], plain[-1] / kw["factor"], rel_tol=1e-12)
    if kw.get("scaling") == "parts":
        plain = np.array(etc.Rotary(dim, base=kw.get("base", 1e4)).freq)
        turns = kw["length"] * plain / (2 * np.pi)
        assert np.allclose(got[turns >= kw["high"]], plain[turns >= kw["high"]], rtol=1e-15)
        assert np.allclose(got[turns <= kw["low"]], plain[turns <= kw["low"]] / kw["factor"], rtol=1e-13)


@pytest.mark.parametrize("bad", (dict(dim=0), dict(dim=3), dict(dim=-2), dict(dim=258), dict(base=0.0), dict(base=-1.0), dict(base=NAN),
                                 dict(base=INF), dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=NAN),
                                 dict(scaling="base", factor=-1.0), dict(scaling="parts"), dict(scaling="parts", length=-1.0),
                                 dict(scaling="parts", length=4096.0, low=4.0, high=4.0), dict(scaling="parts", length=4096.0, high=INF),
                                 dict(layout="pairs"), dict(scaling="other"), dict(freq=[1.0]), dict(base=1e-300, dim=256, scaling="linear", factor=1e-20)))
def test_rotary_object_refuses(bad):
    with pytest.raises((ValueError, etc.EtcError)):
        etc.Rotary(**{**dict(dim=64), **bad})


def test_rotary_fields():
    r = etc.Rotary(8, layout="interleaved", scale=0.5, freq=[1.0, 2.0, 3.0, 4.0])
    assert r.freq == [1.0, 2.0, 3.0, 4.0] and (r._desc.scale, r._desc.pairs, r._desc.layout) == (0.5, 4, 1)


# ---- what the binding hands over ----

class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda packed, stream: self.calls.append((name, packed)) or etc.OK


@pytest.fixture
def calls(monkeypatch):
    library = Recorder()
    monkeypatch.setattr(etc, "_lib", library)
    monkeypatch.setattr(etc, "_device_of", lambda x, what: x.get_device())
    return library.calls


BF16 = torch.bfloat16


def test_strides_of_8_bit_matrices(calls):
    """Data and scales that are slices of larger tensors, in the order of the struct."""
    data, scale = torch.zeros(6, 100, dtype=torch.int8), torch.zeros(6, 9)
    x = torch.zeros(6, 70, dtype=BF16)
    etc.etc_store8(x, etc.Matrix8(data[:, 3:73], scale[:, 1:4], 32), stream=0)
    etc.etc_store8(x, etc.Matrix8(data[:, 3:73], scale[:, 2]), stream=0)
    etc.etc_store8(x[:1], etc.Matrix8(data[:1, 3:73], scale[:1, 2]), stream=0)
    etc.etc_store8(x, etc.Matrix8(data[:, :70].contiguous().view(torch.float8_e4m3fn), torch.zeros(6, 1)), stream=0)
    got = [etc._STORE8.unpack(packed)[7:] for _, packed in calls]
    assert got[0] == (data.data_ptr() + 3, scale.data_ptr() + 4, 6, 70, 100, 9, I8, 32)
    assert got[1] == (data.data_ptr() + 3, scale.data_ptr() + 8, 6, 70, 100, 9, I8, 0)
    assert got[2][2:6] == (1, 70, 70, 1) and got[3][2:] == (6, 70, 70, 1, E4M3, 0)
    etc.etc_load8(etc.Matrix8(data.view(2, 3, 100), torch.zeros(2, 3, 1)), torch.zeros(2, 3, 100), stream=0)
    assert etc._LOAD8.unpack(calls[-1][1])[2:10] == (6, 100, 100, 1, I8, 0, *etc._LOAD8.unpack(calls[-1][1])[8:10])


def test_the_binding_refuses(calls):
    x, q = torch.zeros(4, 64, dtype=BF16), torch.zeros(4, 64, dtype=torch.int8)
    w, s, r = x[0].clone(), torch.zeros(4), torch.zeros(4)
    m = etc.Matrix8(q, s)
    wrong = [
        lambda: etc.Matrix8(q, s, 16), lambda: etc.Matrix8(q, s, -1),
        lambda: etc.etc_store8(x, etc.Matrix8(q.view(torch.uint8), s)), lambda: etc.etc_store8(x, etc.Matrix8(q.t(), s)),
        lambda: etc.etc_store8(x, etc.Matrix8(q, s.double())), lambda: etc.etc_store8(x, etc.Matrix8(q, s[:3])),
        lambda: etc.etc_store8(x, etc.Matrix8(q, s, 32)), lambda: etc.etc_store8(x, etc.Matrix8(q, torch.zeros(2, 4).t(), 32)),
        lambda: etc.etc_store8(x, m, col_scale=s), lambda: etc.etc_store8(x, m, col_scale=torch.zeros(64).double()),
        lambda: etc.etc_store8(x.half(), m),
        lambda: etc.etc_norm(x, w), lambda: etc.etc_norm(x, w, out=x, rstd=r[:3]), lambda: etc.etc_norm(x, w, out=x, rstd=r.double()),
        lambda: etc.etc_norm(x, w, out=x, rstd=torch.zeros(8)[::2]), lambda: etc.etc_norm(x, w.half(), out=x),
        lambda: etc.etc_norm_grad(x, x, w, r[:2], x), lambda: etc.etc_norm_grad(x, x, w, r, x, workspace=q.t()),
        lambda: etc.etc_rotary(x, x, torch.zeros(4), etc_rotary(), 16),
        lambda: etc.etc_rotary(x, x, torch.zeros(8, dtype=torch.int64)[::2], etc_rotary(), 16),
    ]
    for k, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            print("not refused:", k)
    # empty tensors, whose address is 0, where a matrix with elements is due
    e, e8 = x[:0], etc.Matrix8(q[:0], s[:0])
    for name, call in (("residual", lambda: etc.etc_norm(x, w, out=x, residual=e)), ("sum", lambda: etc.etc_norm(x, w, out=x, sum=e)),
                       ("out", lambda: etc.etc_norm(x, w, out=e)), ("out8", lambda: etc.etc_norm(x, w, out=x, out8=e8)),
                       ("dsum", lambda: etc.etc_norm_grad(x, x, w, r, x, dsum=e)), ("x", lambda: etc.etc_norm_grad(x, e8, w, r, x)),
                       ("dweight", lambda: etc.etc_norm_grad(x, x, w, r, x, dweight=r[:0])),
                       ("bias", lambda: etc.etc_matmul8(m, m, torch.zeros(4, 4), bias=r[:0]))):
        with pytest.raises(ValueError, match=name):
            call()
    assert not calls


def etc_rotary():
    r = etc.Rotary.__new__(etc.Rotary)
    r._at = 0
    return r


# ---- the plain implementation itself ----

def test_norm_gradient_against_differences():
    """In 64 bits: the gradients of sum(c * norm) and of sum(d * sum), with respect to x and weight, against central
    differences, whose error is of the order of step^2 and of 2^-52 / step."""
    rng = np.random.default_rng(1)
    x, w, c, d = (rng.standard_normal(s) for s in ((3, 7), (7,), (3, 7), (3, 7)))
    eps, h = 1e-3, 1e-5

    def value(x, w):
        y = block_ref.norm(x, w, None, eps)
        return (c * y["out"][0]).sum() + (d * x).sum()

    r = block_ref.norm(x, w, None, eps)["rstd"][0]
    got = block_ref.norm_grad(c, x, w, r, d, np.zeros(7))
    for i in range(3):
        for j in range(7):
            e = np.zeros((3, 7))
            e[i, j] = h
            assert abs((value(x + e, w) - value(x - e, w)) / (2 * h) - got["dx"][0][i, j]) < 1e-8
    for j in range(7):
        e = np.zeros(7)
        e[j] = h
        assert abs((value(x, w + e) - value(x, w - e)) / (2 * h) - got["dweight"][0][j]) < 1e-8


def test_e4m3_against_torch():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(codes, block_ref.E4M3.astype(np.float32), equal_nan=True)
    v = np.random.default_rng(0).standard_normal(20000).astype(np.float32) * 60
    v = np.concatenate([v, v * 1e-4, ((block_ref.E4M3[:126] + block_ref.E4M3[1:127]) / 2).astype(np.float32)]).clip(-448, 448)
    got = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(got, block_ref.nearest_e4m3(v.astype(np.float64)))


@pytest.mark.parametrize("mistake", ("scale", "data", "largest"))
def test_check_of_8_bits_sees_mistakes(mistake):
    """check_norm8 accepts what the definition gives and refuses a scale or one datum that is a step off."""
    rng = np.random.default_rng(3)
    want = block_ref.norm(rng.standard_normal((4, 100)), rng.standard_normal(100))["out"]
    for eight in ("i8", "e4m3"):
        data, scale = block_ref.store8(want[0].astype(np.float32), eight, 0)
        block_ref.check_norm8(data, scale[:, 0].astype(np.float64), eight, want)
        bad, s = data.copy(), scale[:, 0].astype(np.float64)
        k = int(np.abs(want[0][2]).argmax())
        if mistake == "scale":
            s[1] *= 1 + 1e-4
        elif mistake == "data":
            bad[2, (k + 1) % 100] += 2 if eight == "i8" else 1
        else:
            bad[2, k] -= 1
        with pytest.raises(AssertionError):
            block_ref.check_norm8(bad, s, eight, want)
