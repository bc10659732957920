"""The operators around the projections of a Llama block, with activations in 8
bits, as timed cases.

In front of each projection stands the norm, with the residual's addition; the
projection's product can take its input and weight in 8-bit integers; the query
and key heads that come out of it turn by their positions; and what the backward
pass needs can be kept in 8 bits meanwhile.  `op` says which operator a case calls:

  norm       s = x + residual; out = s * r * weight, r = 1 / sqrt(mean of s^2 + eps); out in x's type or in 8 bits
  norm_grad  dx = dsum + r (dn - n mean(dn n)) with n = x r, dn = weight * grad; the weight's fp32 gradient (a sum
             over rows); x in its type or as it was kept in 8 bits
  keep8      an activation into 8 bits with scales, and back, in bf16
  matmul8    out[m, n] = sx[m] sw[n] * the sum over k of x[m, k] w[n, k] + bias[n], x and w in int8
  rotary     pairs of columns of each head turned by position * frequency, or, for the gradient, turned back

What 8 bits stand for: value = scale * data, one fp32 scale for a row (group 0) or
for `group` columns of it; with a = the largest magnitude there (at least 2^-100),
int8: scale = a / 127, data = x * (127 / a) rounded to nearest even; e4m3 likewise
with 448.  A scale is NaN, and its data 0, where x holds an infinity or NaN.

Sizes come from the model shapes of this repository: tiny GPT (hidden 256),
GPT-1.3B (2048), Llama-7B (hidden 4096, FFN 11008, 32 heads), Llama-70B (8192,
64 query and 8 key and value heads of 128 columns) and odd ones.
"""
import math

import torch

own = False  # False: the plain forms below; True: the library's operators

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}
TOP = {"i8": 127.0, "e4m3": 448.0}
DTYPES8 = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
LEAST = 2.0 ** -100
EPS = 1e-5
DEV = "cuda"


# ---------------------------------------------------------------------------
# The cases

def _norm(name, rows, cols, dtype="bf16", residual=True, eight="", more=0):
    return dict(op="norm", name=name, rows=rows, cols=cols, dtype=dtype, residual=residual, eight=eight, more=more)


def _norm_grad(name, rows, cols, dtype="bf16", kept="", group=0, dsum=True, add=True, more=0):
    return dict(op="norm_grad", name=name, rows=rows, cols=cols, dtype=dtype, kept=kept, group=group, dsum=dsum,
                add=add, more=more)


def _keep8(name, rows, cols, eight="i8", group=128, dtype="bf16", more=0):
    return dict(op="keep8", name=name, rows=rows, cols=cols, eight=eight, group=group, dtype=dtype, more=more)


def _matmul8(name, m, n, k, dtype="bf16", bias=False, more=0):
    return dict(op="matmul8", name=name, m=m, n=n, k=k, dtype=dtype, bias=bias, more=more)


def _rotary(name, tokens, heads, head_dim, dim=None, layout="half", dtype="bf16", others=0, far=2048, scaling="",
            factor=1.0, back=False, ids="int64"):
    return dict(op="rotary", name=name, tokens=tokens, heads=heads, head_dim=head_dim, dim=dim or head_dim,
                layout=layout, dtype=dtype, others=others, far=far, scaling=scaling, factor=factor, back=back, ids=ids)


def listed():
    return [
        # a single token in a 7 B Llama, as when answering: nothing but latency
        _norm("norm-7b-1-token", 1, 4096),
        # the 7 B Llama's step, two sequences of 4096: the sum, and the norm in 8 bits for the products and the
        # weights' gradients, read back as the backward pass reads it
        _norm("norm8-7b-step", 2 * 4096, 4096, eight="i8"),
        # its backward from the activation kept in 8 bits, the residual's gradient and earlier micro-batches' added
        _norm_grad("norm-grad-7b-step", 2 * 4096, 4096, kept="i8", group=128),
        # a backward of odd width, in 32 bits, from the activation itself
        _norm_grad("norm-grad-ragged", 1021, 681, dtype="f32", dsum=False),
        # one sequence of the tiny GPT kept in 8 bits and read back
        _keep8("keep8-tiny", 128, 256),
        # an activation of the 70 B Llama's step, two sequences
        _keep8("keep8-70b-step", 2 * 4096, 8192, eight="e4m3"),
        # a token's query, key and value heads in a 7 B Llama: the weights are read once, nothing else counts
        _matmul8("matmul8-7b-1-token", 1, 3 * 4096, 4096),
        # a batch of answers, one token each, on one of eight ranks of the 70 B Llama: query, key and value heads
        _matmul8("matmul8-70b-batch", 67, 1280, 8192),
        # the 7 B Llama's step, gate and up projections side by side: matrix instructions
        _matmul8("matmul8-7b-step", 2 * 4096, 2 * 11008, 4096),
        # a token's query and key heads in a 7 B Llama
        _rotary("rotary-7b-1-token", 1, 64, 128, far=4096),
        # the 70 B Llama's step, two sequences, query and key heads of rows that hold the value heads too; a context
        # stretched eightfold
        _rotary("rotary-70b-step", 2 * 4096, 72, 128, others=8, far=32768, scaling="parts", factor=8.0),
        # the gradient where a part of each head turns, columns 2 j and 2 j + 1 together, of an odd number of tokens, in 32 bits
        _rotary("rotary-grad-ragged", 1021, 9, 80, dim=52, layout="interleaved", dtype="f32", back=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng):
    """A hidden size: one of the repository's models' or shards', or any, odd ones among them."""
    return rng.choice((256, 504, 681, 2048, 2688, 4096, 5120, 8192, _log_int(rng, 17, 8192), _log_int(rng, 17, 8192)))


def _rows(rng, width):
    return _log_int(rng, 1, max(2, min(16384, (1 << 25) // width)))


def draw(rng):
    op = rng.choice(("norm", "norm_grad", "keep8", "matmul8", "rotary"))
    dtype, more, eight = rng.choice(("bf16", "bf16", "f32")), rng.choice((0, 0, 8, 3)), rng.choice(("i8", "e4m3"))
    group = rng.choice((0, 32, 64, 128, 256))
    if op == "matmul8":
        m = _log_int(rng, 1, 8192)
        n = rng.choice((1280, 2048, 4096, 11008, 12288, _log_int(rng, 16, 22016), _log_int(rng, 16, 22016)))
        k = rng.choice((2048, 4096, 8192, 11008, _log_int(rng, 16, 28672), _log_int(rng, 16, 28672)))
        while n * k > 1 << 27 or m * n * k > 1 << 38:
            n = max(1, n // 2)
        case = _matmul8("", m, n, k, dtype, rng.random() < 0.4, rng.choice((0, 0, 16, 3)))
    elif op == "rotary":
        head_dim = rng.choice((64, 80, 128, 128, 256, rng.randint(2, 256)))
        heads = _log_int(rng, 1, 72)
        tokens = _log_int(rng, 1, max(2, min(16384, (1 << 25) // (heads * head_dim))))
        dim = head_dim // 2 * 2 if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2)
        scaling = rng.choice(("", "", "linear", "base", "parts"))
        if scaling == "base" and dim < 4:  # its exponent, dim / (dim - 2), needs two pairs
            scaling = ""
        case = _rotary("", tokens, heads, head_dim, dim, rng.choice(("half", "interleaved")), dtype,
                       rng.choice((0, 0, 1, 8)), rng.choice((128, 4096, 131072, 1 << 20)), scaling,
                       rng.choice((2.0, 8.0, 32.0)) if scaling else 1.0, rng.random() < 0.4, rng.choice(("int64", "int32")))
    else:
        cols = _width(rng)
        rows = _rows(rng, cols)
        if op == "norm":
            case = _norm("", rows, cols, dtype, rng.random() < 0.7, rng.choice(("", "", eight)), more)
        elif op == "norm_grad":
            case = _norm_grad("", rows, cols, dtype, rng.choice(("", eight)), group, rng.random() < 0.7,
                              rng.random() < 0.5, more)
        else:
            case = _keep8("", rows, cols, eight, group, dtype, more)
    return {k: v for k, v in case.items() if k != "name"}


# ---------------------------------------------------------------------------
# Inputs

def _normal(gen, rows, cols, dtype, std=1.0, more=0):
    """[rows, cols] values in rows of cols + more elements, as a slice of a fused buffer is."""
    full = torch.empty(rows, cols + more, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=gen)
    return full.to(dtype)[:, :cols]


def _activation(gen, rows, cols, dtype, more=0):
    """As a residual stream is: one channel in a hundred is ten times as large as the others."""
    x = torch.empty(rows, cols + more, dtype=torch.float32, device=DEV).normal_(0.0, 1.0, generator=gen)
    x *= torch.where(torch.rand(cols + more, generator=gen, device=DEV) < 0.01, 10.0, 1.0)
    return x.to(dtype)[:, :cols]


def _groups(cols, group):
    return -(-cols // group) if group else 1


def _to8(x, eight, group):
    """fp32 x in 8 bits: (data, scales [rows, groups])."""
    rows, cols = x.shape
    n, width = _groups(cols, group), group or cols
    y = torch.nn.functional.pad(x, (0, n * width - cols)).view(rows, n, width)
    a = y.abs().amax(-1, keepdim=True)
    good = torch.isfinite(a)
    a = a.clamp(min=LEAST)
    q = torch.where(good, y * (TOP[eight] / a), 0.0)
    q = (q.round() if eight == "i8" else q).to(DTYPES8[eight])
    scale = torch.where(good, a / TOP[eight], math.nan)
    return q.view(rows, -1)[:, :cols], scale.view(rows, n)


def _from8(data, scale, group):
    """The fp32 values of data with scales [rows, groups]."""
    wide = scale.repeat_interleave(group, 1)[:, :data.shape[1]] if group else scale
    return data.float() * wide


def _strided(x, more):
    """x in rows of `more` elements more."""
    full = torch.zeros(x.shape[0], x.shape[1] + more, dtype=x.dtype, device=DEV)
    full[:, :x.shape[1]].copy_(x)
    return full[:, :x.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    s = dict(case=case, op=op)
    if op == "matmul8":
        x, sx = _to8(_activation(gen, case["m"], case["k"], torch.float32), "i8", 0)
        w, sw = _to8(_normal(gen, case["n"], case["k"], torch.float32, 0.02), "i8", 0)
        s["x"], s["sx"], s["w"], s["sw"] = _strided(x, case["more"]), sx.view(-1), w.contiguous(), sw.view(-1)
        s["bias"] = _normal(gen, 1, case["n"], DTYPES[case["dtype"]])[0] if case["bias"] else None
        s["out"] = torch.empty(case["m"], case["n"], dtype=DTYPES[case["dtype"]], device=DEV)
        return s
    t = DTYPES[case["dtype"]]
    if op == "rotary":
        cols = case["heads"] * case["head_dim"]
        s["x"] = _normal(gen, case["tokens"], cols, t, more=case["others"] * case["head_dim"])
        s["positions"] = torch.randint(0, case["far"], (case["tokens"],), generator=gen, device=DEV)
        if case["tokens"] > 1:  # a sequence somewhere in its context; one token: as it comes
            start = int(seed) % max(1, case["far"] - case["tokens"])
            s["positions"] = (start + torch.arange(case["tokens"], device=DEV)) % case["far"]
        s["positions"] = s["positions"].to(getattr(torch, case["ids"]))
        s["freq"], s["scale"] = _frequencies(case)
        s["out"] = torch.empty(case["tokens"], cols, dtype=t, device=DEV)
        return s
    rows, cols = case["rows"], case["cols"]
    s["x"] = _activation(gen, rows, cols, t, case["more"])
    if op in ("norm", "norm_grad"):
        s["weight"] = (1.0 + 0.1 * torch.randn(cols, generator=gen, device=DEV)).to(t)
    if op == "norm":
        s["residual"] = _activation(gen, rows, cols, t) if case["residual"] else None
        s["sum"] = torch.empty(rows, cols, dtype=t, device=DEV) if case["residual"] else None
        # what 8 bits stand for is read back in bf16, the type that products take it in
        s["out"] = torch.empty(rows, cols, dtype=torch.bfloat16 if case["eight"] else t, device=DEV)
        s["rstd"] = torch.empty(rows, device=DEV)
    elif op == "norm_grad":
        s["grad"] = _normal(gen, rows, cols, t)
        s["dsum"] = _normal(gen, rows, cols, t) if case["dsum"] else None
        s["rstd"] = torch.rsqrt(s["x"].float().square().mean(-1) + EPS)
        s["dx"] = torch.empty(rows, cols, dtype=t, device=DEV)
        s["dweight"] = _normal(gen, 1, cols, torch.float32)[0]
        if case["kept"]:
            data, scale = _to8(s.pop("x").float(), case["kept"], case["group"])
            s["data"], s["scale"] = data.contiguous(), scale.contiguous()
    else:
        s["out"] = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    eight = case.get("eight")
    if eight:
        s["data"] = torch.empty(rows, cols, dtype=DTYPES8[eight], device=DEV)
        s["scale"] = torch.empty(rows, _groups(cols, case.get("group", 0)), device=DEV)
    return s


BASE, LENGTH, LOW, HIGH = 10000.0, 4096.0, 1.0, 32.0


def _frequencies(case):
    """Radians a position of each pair, in 64 bits on the host as a model's configuration gives them, and what sine
    and cosine are multiplied with."""
    d, f = case["dim"], case["factor"]
    base = BASE * f ** (d / (d - 2)) if case["scaling"] == "base" else BASE
    freq = torch.tensor([base ** (-2 * j / d) for j in range(d // 2)], dtype=torch.float64, device=DEV)
    if case["scaling"] == "linear":
        freq = freq / f
    if case["scaling"] == "parts":
        keep = ((LENGTH * freq / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        freq = freq * (keep + (1 - keep) / f)
        return freq, 0.1 * math.log(f) + 1.0
    return freq, 1.0


# ---------------------------------------------------------------------------
# The plain forms

def _plain_norm(s):
    case = s["case"]
    x = s["x"].float()
    if case["residual"]:
        x = x + s["residual"].float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    y = x * r * s["weight"].float()
    if case["eight"]:
        y = _from8(*_to8(y, case["eight"], 0), 0)
    out = [y.to(s["out"].dtype), r.view(-1)]
    return out + [x.to(s["sum"].dtype)] if case["residual"] else out


def _plain_norm_grad(s):
    case = s["case"]
    x = _from8(s["data"], s["scale"], case["group"]) if case["kept"] else s["x"].float()
    n, g = x * s["rstd"][:, None], s["grad"].float()
    dn = g * s["weight"].float()
    dx = s["rstd"][:, None] * (dn - n * (dn * n).mean(-1, keepdim=True))
    if case["dsum"]:
        dx = dx + s["dsum"].float()
    d = (g * n).sum(0)
    return [dx.to(s["dx"].dtype), s["dweight"].add_(d) if case["add"] else s["dweight"].copy_(d)]


def _plain_keep8(s):
    case = s["case"]
    return _from8(*_to8(s["x"].float(), case["eight"], case["group"]), case["group"]).to(s["out"].dtype)


def _plain_matmul8(s):
    y = s["x"].float() @ s["w"].float().t()
    y = y * s["sx"][:, None] * s["sw"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["out"].dtype)


def _plain_rotary(s):
    case = s["case"]
    d, h = case["dim"], case["dim"] // 2
    angle = s["positions"].double()[:, None] * s["freq"]
    c, n = ((f(angle) * s["scale"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    if case["back"]:
        n = -n
    x = s["x"].float().reshape(case["tokens"], case["heads"], case["head_dim"])
    out = x.clone()
    a, b = (x[..., :h], x[..., h:d]) if case["layout"] == "half" else (x[..., 0:d:2], x[..., 1:d:2])
    u, v = (out[..., :h], out[..., h:d]) if case["layout"] == "half" else (out[..., 0:d:2], out[..., 1:d:2])
    u.copy_(a * c - b * n)
    v.copy_(b * c + a * n)
    return out.view(case["tokens"], -1).to(s["out"].dtype)


# ---------------------------------------------------------------------------
# The library's operators

def _eight(etc, s, group):
    """The 8-bit matrix of the state's data and scales, which a program keeps with its buffers."""
    if "matrix8" not in s:
        s["matrix8"] = etc.Matrix8(s["data"], s["scale"], group=group)
    return s["matrix8"]


def _own(s):
    from paper_2607_04749_amd import etc
    case, op = s["case"], s["op"]
    if op == "norm":
        if case["eight"]:
            q = _eight(etc, s, 0)
            etc.etc_norm(s["x"], s["weight"], out8=q, residual=s["residual"], sum=s["sum"], rstd=s["rstd"], eps=EPS)
            etc.etc_load8(q, s["out"])
        else:
            etc.etc_norm(s["x"], s["weight"], out=s["out"], residual=s["residual"], sum=s["sum"], rstd=s["rstd"], eps=EPS)
        out = [s["out"], s["rstd"]]
        return out + [s["sum"]] if case["residual"] else out
    if op == "norm_grad":
        if "work" not in s:  # scratch memory that a training loop keeps from step to step
            s["work"] = torch.empty(etc.etc_norm_grad_bytes(case["rows"], case["cols"]), dtype=torch.uint8, device=DEV)
        x = _eight(etc, s, case["group"]) if case["kept"] else s["x"]
        etc.etc_norm_grad(s["grad"], x, s["weight"], s["rstd"], s["dx"], dsum=s["dsum"], dweight=s["dweight"],
                          workspace=s["work"], accumulate=case["add"])
        return [s["dx"], s["dweight"]]
    if op == "keep8":
        q = _eight(etc, s, case["group"])
        etc.etc_store8(s["x"], q)
        etc.etc_load8(q, s["out"])
        return s["out"]
    if op == "matmul8":
        if "x8" not in s:
            s["x8"], s["w8"] = etc.Matrix8(s["x"], s["sx"]), etc.Matrix8(s["w"], s["sw"])
        etc.etc_matmul8(s["x8"], s["w8"], s["out"], bias=s["bias"])
        return s["out"]
    if "rotary" not in s:  # a model has one for all its layers
        more = dict(factor=case["factor"], scaling=case["scaling"] or None)
        if case["scaling"] == "parts":
            more.update(length=LENGTH, low=LOW, high=HIGH, scale=s["scale"])
        s["rotary"] = etc.Rotary(case["dim"], base=BASE, layout=case["layout"], **more)
    etc.etc_rotary(s["x"], s["out"], s["positions"], s["rotary"], case["head_dim"], backward=case["back"])
    return s["out"]


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "keep8": _plain_keep8, "matmul8": _plain_matmul8,
         "rotary": _plain_rotary}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without

def work(case):
    op, e = case["op"], ESIZE[case["dtype"]]
    if op == "matmul8":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + m * n * e + 4 * (m + n) + (n * e if case["bias"] else 0), "flops": 2 * m * n * k}
    if op == "rotary":
        n = case["tokens"] * case["heads"] * case["head_dim"]
        return {"bytes": 2 * n * e + case["tokens"] * (8 if case["ids"] == "int64" else 4),
                "flops": 3 * case["tokens"] * case["heads"] * case["dim"]}
    rows, cols = case["rows"], case["cols"]
    n = rows * cols
    if op == "keep8":  # to 8 bits and back
        return {"bytes": n * (e + 4) + 8 * rows * _groups(cols, case["group"]), "flops": 4 * n}
    if op == "norm":
        moved = n * e * (3 if case["residual"] else 1) + (4 * n + 8 * rows if case["eight"] else n * e)
        return {"bytes": moved + cols * e + 4 * rows, "flops": 6 * n}
    kept = n + 4 * rows * _groups(cols, case["group"]) if case["kept"] else n * e
    return {"bytes": n * e * (3 if case["dsum"] else 2) + kept + cols * (e + 4 * (1 + case["add"])) + 4 * rows,
            "flops": 11 * n}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits

def _nearest8(v, eight):
    """64-bit values in -TOP .. TOP to the nearest that 8 bits hold, ties to even."""
    if eight == "i8":
        return torch.round(v)
    # steps of 2^-3 of the leading bit, of 2^-9 below 2^-6
    _, exponent = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (exponent - 1).clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _through8(x, eight, group):
    """64-bit x as its 8 bits stand for it, slice by slice of columns."""
    out = torch.empty_like(x)
    width = group or x.shape[1]
    for c in range(0, x.shape[1], width):
        part = x[:, c:c + width]
        unit = part.abs().max(1, keepdim=True).values.clamp(min=LEAST) / TOP[eight]
        out[:, c:c + width] = _nearest8(part / unit, eight) * unit
    return out


def _turned(s):
    """Each pair as a complex number, times e^(i position freq), its conjugate for the gradient."""
    case = s["case"]
    tokens, heads, width, d = case["tokens"], case["heads"], case["head_dim"], case["dim"]
    x = s["x"].double().reshape(tokens, heads, width)
    turn = torch.polar(torch.full((), s["scale"], dtype=torch.float64, device=DEV),
                       s["positions"].double().view(-1, 1, 1) * s["freq"].view(1, 1, -1))
    turn = turn.conj() if case["back"] else turn
    if case["layout"] == "interleaved":
        z = torch.view_as_complex(x[..., :d].reshape(tokens, heads, d // 2, 2).contiguous()) * turn
        done = torch.view_as_real(z).reshape(tokens, heads, d)
    else:
        z = torch.complex(x[..., :d // 2], x[..., d // 2:d]) * turn
        done = torch.cat((z.real, z.imag), -1)
    return torch.cat((done, x[..., d:]), -1).reshape(tokens, heads * width)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotary":
        return _turned(s)
    if op == "matmul8":
        y = torch.mm(s["x"].double() * s["sx"].double().unsqueeze(1), (s["w"].double() * s["sw"].double().unsqueeze(1)).t())
        return y if s["bias"] is None else y + s["bias"].double()
    if op == "keep8":
        return _through8(s["x"].double(), case["eight"], case["group"])
    if op == "norm":
        x = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
        size = torch.linalg.vector_norm(x, dim=1)
        r = 1.0 / torch.sqrt(size * size / case["cols"] + EPS)
        y = torch.einsum("ij,i,j->ij", x, r, s["weight"].double())
        y = _through8(y, case["eight"], 0) if case["eight"] else y
        return [y, r, x] if case["residual"] else [y, r]
    r = s["rstd"].double()
    if case["kept"]:
        scale, width = s["scale"].double(), case["group"] or case["cols"]
        x = torch.stack([s["data"][:, c].double() * scale[:, c // width] for c in range(case["cols"])], 1)
    else:
        x = s["x"].double()
    g, w = s["grad"].double(), s["weight"].double()
    # each row's gradient less its part along the row: r w g - r^3 x <x, w g> / cols
    along = torch.einsum("ij,j,ij->i", x, w, g) * r ** 3 / case["cols"]
    dx = torch.einsum("i,j,ij->ij", r, w, g) - along.unsqueeze(1) * x
    dw = torch.einsum("ij,i,ij->j", g, r, x)
    return [dx + s["dsum"].double() if case["dsum"] else dx, dw + s["dweight"].double() if case["add"] else dw]
