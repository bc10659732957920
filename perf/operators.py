"""The operators of a training step on the states that this library moves, as
timed cases.

A rank on the first pipeline stage looks its tokens up in its share of the
vocabulary (and, in a GPT, adds positions), every block ends in bias, dropout
and residual, the backward pass brings the gradients of both back, and Adam
turns the gradients into the bf16 parameter, fp32 master, m and v that a
migration moves.  `op` says which operator a case calls:

  embed         out = drop(scale * table[id] + pos_table[position])
  embed_grad    the table's fp32 gradient, by sorted tokens
  dropout       out = residual + drop(x + bias)
  dropout_grad  dx, and the bias's fp32 gradient (a sum over rows)
  adam          one step over a range of the four arenas

The random numbers of dropout are a function of (seed, call, row, column):
16 bits per element from Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
"Parallel Random Numbers: As Easy as 1, 2, 3", SC 2011).  An element is dropped
where its 16 bits are below t = floor(65536 p + 1/2), and scaled by
65536 / (65536 - t) elsewhere.

Sizes come from the model shapes of this repository: tiny GPT (hidden 256,
vocabulary 1024, 128 positions), GPT-1.3B (2048, 50304, 2048), Llama-7B (4096,
32000), Llama-70B (8192, 32000) and the two of odd widths of perf/cases.py.
"""
import math

import numpy as np
import torch

own = False  # False: the plain forms below; True: the library's operators

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}
DEV = "cuda"


# ---------------------------------------------------------------------------
# The cases

def _embed(name, tokens, hidden, vocab, rows=None, row0=0, pos=0, scale=1.0, p=0.0, table="bf16", out="bf16",
           pad=0.0, ids="int64"):
    return dict(op="embed", name=name, tokens=tokens, hidden=hidden, vocab=vocab, rows=rows or vocab, row0=row0,
                pos=pos, scale=scale, p=p, table=table, out=out, pad=pad, ids=ids)


def _embed_grad(name, tokens, hidden, vocab, rows=None, row0=0, scale=1.0, p=0.0, grad="bf16", add=True, pad=0.0,
                ids="int64"):
    return dict(op="embed_grad", name=name, tokens=tokens, hidden=hidden, vocab=vocab, rows=rows or vocab, row0=row0,
                scale=scale, p=p, grad=grad, add=add, pad=pad, ids=ids)


def _dropout(name, rows, cols, p=0.1, dtype="bf16", bias=True, residual=True, more=0):
    return dict(op="dropout", name=name, rows=rows, cols=cols, p=p, dtype=dtype, bias=bias, residual=residual,
                more=more)


def _dropout_grad(name, rows, cols, p=0.1, dtype="bf16", bias=True, add=True, more=0):
    return dict(op="dropout_grad", name=name, rows=rows, cols=cols, p=p, dtype=dtype, bias=bias, add=add, more=more)


def _adam(name, count, first=0, decay=0.01, clip=True):
    return dict(op="adam", name=name, count=count, first=first, decay=decay, clip=clip)


def listed():
    return [
        # a single token in a 7 B Llama, as when answering: nothing but latency
        _embed("embed-7b-1-token", 1, 4096, 32000),
        # the input of a 1.3 B GPT's step, eight sequences: lookup, positions and dropout at once
        _embed("embed-1.3b-step", 8 * 2048, 2048, 50304, pos=2048, scale=math.sqrt(2048.0), p=0.1),
        # one of eight shares of a 70 B Llama's vocabulary: most tokens belong to other ranks
        _embed("embed-70b-shard", 2 * 4096, 8192, 32000, rows=4000, row0=12000, ids="int32"),
        # the smallest gradient in use: one sequence of tiny GPT, the table's gradient written whole
        _embed_grad("embed-grad-tiny", 128, 256, 1024, p=0.1, add=False),
        # the gradient of the 1.3 B GPT's step, added to that of the micro-batches before
        _embed_grad("embed-grad-1.3b-step", 8 * 2048, 2048, 50304, scale=math.sqrt(2048.0), p=0.1),
        # a quarter of a 7 B Llama's vocabulary, padded sequences, the first micro-batch: the gradient written whole
        _embed_grad("embed-grad-7b-shard", 2 * 4096, 4096, 32000, rows=8000, row0=0, add=False, pad=0.05),
        # a block's epilogue in tiny GPT: one sequence
        _dropout("dropout-tiny", 128, 256),
        # a block's epilogue in the 1.3 B GPT, eight sequences
        _dropout("dropout-1.3b-step", 8 * 2048, 2048),
        # the backward of an epilogue of odd width, in 32 bits
        _dropout_grad("dropout-grad-ragged", 1021, 681, dtype="f32"),
        # the backward of the 1.3 B GPT's epilogue, the bias's gradient added to earlier ones
        _dropout_grad("dropout-grad-1.3b-step", 8 * 2048, 2048),
        # Adam over a rank of tiny GPT (TP 4): the whole arena
        _adam("adam-tiny", 893440),
        # Adam over a rank of the 1.3 B GPT (TP 4, PP 2): the whole arena
        _adam("adam-1.3b-rank", 181135360),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng):
    """A hidden size: one of the repository's models' or shards', or any, odd ones among them."""
    return rng.choice((256, 504, 681, 2048, 2688, 4096, 5120, 8192, _log_int(rng, 17, 8192), _log_int(rng, 17, 8192)))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "dropout", "dropout_grad", "adam"))
    if op == "adam":
        return {k: v for k, v in _adam("", _log_int(rng, 1000, 180_000_000), rng.choice((0, 0, 128, 1003)),
                                       rng.choice((0.0, 0.01, 0.1)), rng.random() < 0.7).items() if k != "name"}
    width = _width(rng)
    rows = _log_int(rng, 1, max(2, min(16384, (1 << 25) // width)))
    p = rng.choice((0.0, 0.1, 0.1, 0.25, round(rng.uniform(0.01, 0.6), 3)))
    if op == "dropout":
        case = _dropout("", rows, width, p, rng.choice(("bf16", "f32")), rng.random() < 0.7, rng.random() < 0.7,
                        rng.choice((0, 0, 8, 3)))
    elif op == "dropout_grad":
        case = _dropout_grad("", rows, width, p, rng.choice(("bf16", "f32")), rng.random() < 0.7, rng.random() < 0.5,
                             rng.choice((0, 0, 8, 3)))
    else:
        vocab = rng.choice((1024, 5004, 32000, 50268, 50304, _log_int(rng, 300, 131072)))
        while vocab * width > 1 << 27:
            vocab //= 2
        shards = rng.choice((1, 1, 2, 4, 8))
        more = dict(rows=vocab // shards, row0=rng.randrange(shards) * (vocab // shards),
                    scale=rng.choice((1.0, math.sqrt(width))), p=p, pad=rng.choice((0.0, 0.0, 0.05, 0.4)),
                    ids=rng.choice(("int64", "int32")))
        if op == "embed":
            case = _embed("", rows, width, vocab, pos=rng.choice((0, 128, 1000, 2048)),
                          table=rng.choice(("bf16", "bf16", "f32")), out=rng.choice(("bf16", "bf16", "f32")), **more)
        else:
            case = _embed_grad("", rows, width, vocab, grad=rng.choice(("bf16", "bf16", "f32")),
                               add=rng.random() < 0.5, **more)
    return {k: v for k, v in case.items() if k != "name"}


# ---------------------------------------------------------------------------
# Inputs

def _tokens(case, gen):
    """Ids over the whole vocabulary, frequent ones low as a tokenizer numbers
    them (P(id) ~ 1 / (id + 1)); padding is -1, which no rank holds."""
    u = torch.rand(case["tokens"], generator=gen, device=DEV, dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["vocab"] + 1)) - 1).long().clamp_(0, case["vocab"] - 1)
    if case["pad"]:
        ids[torch.rand(case["tokens"], generator=gen, device=DEV) < case["pad"]] = -1
    return ids.to(getattr(torch, case["ids"]))


def _normal(gen, rows, cols, dtype, std=1.0, more=0):
    """[rows, cols] values in rows of cols + more elements, as a slice of a fused buffer is."""
    full = torch.empty(rows, cols + more, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=gen)
    return full.to(dtype)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    s = dict(case=case, op=op, seed=(0x9E3779B97F4A7C15 * (seed + 1)) % (1 << 63), call=seed % 97)
    if op == "embed":
        s["ids"] = _tokens(case, gen)
        s["table"] = _normal(gen, case["rows"], case["hidden"], DTYPES[case["table"]], 0.02)
        s["pos_table"] = s["positions"] = None
        if case["pos"]:
            s["pos_table"] = _normal(gen, case["pos"], case["hidden"], DTYPES[case["table"]], 0.02)
            s["positions"] = (torch.arange(case["tokens"], device=DEV) % case["pos"]).to(s["ids"].dtype)
        s["out"] = torch.empty(case["tokens"], case["hidden"], dtype=DTYPES[case["out"]], device=DEV)
    elif op == "embed_grad":
        s["ids"] = _tokens(case, gen)
        s["grad"] = _normal(gen, case["tokens"], case["hidden"], DTYPES[case["grad"]])
        s["dtable"] = _normal(gen, case["rows"], case["hidden"], torch.float32)
    elif op == "dropout":
        t = DTYPES[case["dtype"]]
        s["x"] = _normal(gen, case["rows"], case["cols"], t, more=case["more"])
        s["bias"] = _normal(gen, 1, case["cols"], t)[0] if case["bias"] else None
        s["residual"] = _normal(gen, case["rows"], case["cols"], t) if case["residual"] else None
        s["out"] = torch.empty(case["rows"], case["cols"], dtype=t, device=DEV)
    elif op == "dropout_grad":
        t = DTYPES[case["dtype"]]
        s["grad"] = _normal(gen, case["rows"], case["cols"], t, more=case["more"])
        s["dx"] = torch.empty(case["rows"], case["cols"], dtype=t, device=DEV)
        s["dbias"] = _normal(gen, 1, case["cols"], torch.float32)[0] if case["bias"] else None
    else:
        n = case["first"] + case["count"]
        s["master"] = torch.empty(n, device=DEV).normal_(0.0, 0.02, generator=gen)
        s["param"] = s["master"].to(torch.bfloat16)
        s["m"] = torch.empty(n, device=DEV).normal_(0.0, 1e-3, generator=gen)
        s["v"] = torch.empty(n, device=DEV).normal_(0.0, 1e-3, generator=gen).square_()
        s["grad"] = torch.empty(n, device=DEV).normal_(0.0, 1e-3, generator=gen)
        s["clip"] = torch.full((1,), 0.37, device=DEV) if case["clip"] else None
        s["step"] = 1 + seed % 1000
    return s


LR, BETA1, BETA2, EPS = 3e-4, 0.9, 0.999, 1e-8


# ---------------------------------------------------------------------------
# The plain forms

MASK32 = 0xFFFFFFFF


def _keep(s, rows, cols):
    """keep[i, j] of rows x cols, and the scale of what is kept."""
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, device=DEV).repeat(rows, 1)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, blocks)
    c2 = torch.zeros_like(c0)
    c3 = torch.full_like(c0, s["call"])
    k0, k1 = s["seed"] & MASK32, s["seed"] >> 32
    for _ in range(10):  # the generator's rounds; 32 x 32 -> 64 bit products wrap as they should
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & MASK32) ^ c1 ^ k0, b & MASK32, ((a >> 32) & MASK32) ^ c3 ^ k1, a & MASK32
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    words = torch.stack((c0, c1, c2, c3), -1)
    u = torch.stack((words & 0xFFFF, words >> 16), -1).reshape(rows, blocks * 8)[:, :cols]
    t = math.floor(65536 * s["case"]["p"] + 0.5)
    return u >= t, (65536 / (65536 - t) if t < 65536 else 0.0)


def _drop(s, x):
    if s["case"]["p"] == 0:
        return x
    keep, scale = _keep(s, *x.shape)
    return torch.where(keep, x * scale, 0.0)


def _plain_embed(s):
    case = s["case"]
    row = s["ids"].long() - case["row0"]
    held = (row >= 0) & (row < case["rows"])
    x = s["table"][row.clamp(0, case["rows"] - 1)].float() * case["scale"]
    x = torch.where(held[:, None], x, 0.0)
    if case["pos"]:
        x = x + s["pos_table"][s["positions"].long()].float()
    return _drop(s, x).to(s["out"].dtype)


def _plain_embed_grad(s):
    case = s["case"]
    row = s["ids"].long() - case["row0"]
    row = torch.where((row >= 0) & (row < case["rows"]), row, case["rows"])
    g = _drop(s, s["grad"].float())
    d = torch.zeros(case["rows"] + 1, case["hidden"], device=DEV)
    d = d.index_add_(0, row, g)[:-1] * case["scale"]
    return s["dtable"].add_(d) if case["add"] else s["dtable"].copy_(d)


def _plain_dropout(s):
    x = s["x"].float()
    if s["bias"] is not None:
        x = x + s["bias"].float()
    x = _drop(s, x)
    if s["residual"] is not None:
        x = x + s["residual"].float()
    return x.to(s["out"].dtype)


def _plain_dropout_grad(s):
    g = _drop(s, s["grad"].float())
    if s["dbias"] is None:
        return [g.to(s["dx"].dtype)]
    d = g.sum(0)
    return [g.to(s["dx"].dtype), s["dbias"].add_(d) if s["case"]["add"] else s["dbias"].copy_(d)]


def _plain_adam(s):
    case = s["case"]
    w, m, v, p, g = (s[k][case["first"]:] for k in ("master", "m", "v", "param", "grad"))
    if s["clip"] is not None:
        g = g * s["clip"]
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    update = (m / (1 - BETA1 ** s["step"])) / ((v / (1 - BETA2 ** s["step"])).sqrt() + EPS)
    w.sub_((update + w * case["decay"]) * LR)
    p.copy_(w)
    return [s["param"], s["master"], s["m"], s["v"]]


# ---------------------------------------------------------------------------
# The library's operators

def _dropout_of(etc, s):
    if "dropout" not in s:
        s["dropout"] = etc.Dropout(s["case"]["p"], s["seed"], call=s["call"])
    return s["dropout"]


def _workspace(s, nbytes):
    """Scratch memory that a training loop keeps from step to step."""
    if "work" not in s:
        s["work"] = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    return s["work"]


def _own(s):
    from paper_2607_04749_amd import etc
    case, op = s["case"], s["op"]
    if op == "embed":
        etc.etc_embed(s["ids"], s["table"], s["out"], row0=case["row0"], scale=case["scale"],
                      positions=s["positions"], pos_table=s["pos_table"], dropout=_dropout_of(etc, s))
        return s["out"]
    if op == "embed_grad":
        work = s.get("work")
        if work is None:
            work = _workspace(s, etc.etc_embed_grad_bytes(case["tokens"], case["rows"], case["hidden"]))
        etc.etc_embed_grad(s["ids"], s["grad"], s["dtable"], work, row0=case["row0"], scale=case["scale"],
                           dropout=_dropout_of(etc, s), accumulate=case["add"])
        return s["dtable"]
    if op == "dropout":
        etc.etc_dropout(s["x"], s["out"], _dropout_of(etc, s), bias=s["bias"], residual=s["residual"])
        return s["out"]
    if op == "dropout_grad":
        if s["dbias"] is None:
            etc.etc_dropout_grad(s["grad"], s["dx"], _dropout_of(etc, s))
            return [s["dx"]]
        work = s.get("work")
        if work is None:
            work = _workspace(s, etc.etc_dropout_grad_bytes(case["rows"], case["cols"]))
        etc.etc_dropout_grad(s["grad"], s["dx"], _dropout_of(etc, s), dbias=s["dbias"], workspace=work,
                             accumulate=case["add"])
        return [s["dx"], s["dbias"]]
    arenas = [s["param"], s["master"], s["m"], s["v"]]
    etc.etc_adam(arenas, s["grad"], step=s["step"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                 weight_decay=case["decay"], grad_scale=s["clip"], first=case["first"], count=case["count"])
    return arenas


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "dropout": _plain_dropout,
         "dropout_grad": _plain_dropout_grad, "adam": _plain_adam}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without

def _held(case):
    """Expected tokens and distinct rows of this rank's share."""
    v = np.arange(case["row0"], case["row0"] + case["rows"], dtype=np.float64)
    share = np.log((v + 2) / (v + 1)) / math.log(case["vocab"] + 1) * (1 - case["pad"])
    return case["tokens"] * share.sum(), (1 - (1 - share) ** case["tokens"]).sum()


def work(case):
    op = case["op"]
    if op == "adam":
        return {"bytes": 30 * case["count"], "flops": 14 * case["count"]}
    if op in ("embed", "embed_grad"):
        held, distinct = _held(case)
        ids, n = (8 if case["ids"] == "int64" else 4) * case["tokens"], case["tokens"] * case["hidden"]
        if op == "embed":
            read = distinct * case["hidden"] * ESIZE[case["table"]]
            if case["pos"]:
                read += min(case["pos"], case["tokens"]) * case["hidden"] * ESIZE[case["table"]] + ids
            return {"bytes": ids + read + n * ESIZE[case["out"]], "flops": 3 * n}
        table = 8 * distinct if case["add"] else 4 * case["rows"]
        return {"bytes": ids + (held * ESIZE[case["grad"]] + table) * case["hidden"],
                "flops": 2 * held * case["hidden"]}
    n, e = case["rows"] * case["cols"], ESIZE[case["dtype"]]
    if op == "dropout":
        return {"bytes": n * e * (3 if case["residual"] else 2) + (e * case["cols"] if case["bias"] else 0),
                "flops": 3 * n}
    return {"bytes": 2 * n * e + (4 * (1 + case["add"]) * case["cols"] if case["bias"] else 0), "flops": 2 * n}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits

def _factor(s, rows, cols):
    """What each element is multiplied with by dropout: 0 or 1 / (share kept); on the host, in unsigned words."""
    p = s["case"]["p"]
    if p == 0:
        return None
    nb = -(-cols // 8)
    t = int(math.floor(p * 65536.0 + 0.5))
    lo, sh = np.uint64(MASK32), np.uint64(32)
    out = np.empty((rows, cols), np.uint16)
    for a in range(0, rows, 1 + (1 << 20) // nb):
        r = np.arange(a, min(rows, a + 1 + (1 << 20) // nb), dtype=np.uint64)
        x = [np.broadcast_to(np.arange(nb, dtype=np.uint64)[None, :], (r.size, nb)),
             np.broadcast_to((r & lo)[:, None], (r.size, nb)), np.broadcast_to((r >> sh)[:, None], (r.size, nb)),
             np.full((r.size, nb), s["call"], np.uint64)]
        key = [s["seed"] % (1 << 32), s["seed"] // (1 << 32)]
        for _ in range(10):
            u, w = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
            x = [(w >> sh) ^ x[1] ^ np.uint64(key[0]), w & lo, (u >> sh) ^ x[3] ^ np.uint64(key[1]), u & lo]
            key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
        halves = np.stack(x, -1).astype("<u4").view("<u2").reshape(r.size, nb * 8)
        out[a:a + r.size] = halves[:, :cols]
    kept = torch.from_numpy(out >= t) if t < 65536 else torch.zeros(rows, cols, dtype=torch.bool)
    return kept.to(DEV), (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _dropped(s, x):
    f = _factor(s, *x.shape)
    return x if f is None else torch.where(f[0], x * f[1], torch.zeros((), dtype=x.dtype, device=x.device))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        # an extra row of zeros stands for every id that this rank does not hold
        rows = torch.cat((s["table"].double() * case["scale"], torch.zeros(1, case["hidden"], device=DEV).double()))
        k = s["ids"].long() - case["row0"]
        k[(k < 0) | (k >= case["rows"])] = case["rows"]
        x = rows.index_select(0, k)
        if case["pos"]:
            x += s["pos_table"].double().index_select(0, s["positions"].long())
        return _dropped(s, x)
    if op == "embed_grad":
        # sorted ids, running sums, differences at the ends of equal ids
        g = _dropped(s, s["grad"].double())
        k = s["ids"].long() - case["row0"]
        mine = ((k >= 0) & (k < case["rows"])).nonzero().flatten()
        k, order = torch.sort(k[mine])
        sums = torch.cumsum(torch.cat((torch.zeros(1, case["hidden"], device=DEV).double(), g[mine[order]])), 0)
        bounds = torch.searchsorted(k, torch.arange(case["rows"] + 1, device=DEV))
        d = (sums[bounds[1:]] - sums[bounds[:-1]]) * case["scale"]
        return d + s["dtable"].double() if case["add"] else d
    if op == "dropout":
        x = s["x"].double()
        x = _dropped(s, x if s["bias"] is None else x + s["bias"].double())
        return x if s["residual"] is None else x + s["residual"].double()
    if op == "dropout_grad":
        g = _dropped(s, s["grad"].double())
        if s["dbias"] is None:
            return [g]
        return [g, g.sum(0) + (s["dbias"].double() if case["add"] else 0.0)]
    a = case["first"]
    w, m, v = (s[k].double() for k in ("master", "m", "v"))
    g = s["grad"].double()[a:] * (1.0 if s["clip"] is None else s["clip"].double())
    m[a:] += (g - m[a:]) * (1 - BETA1)
    v[a:] += (g * g - v[a:]) * (1 - BETA2)
    mean, var = m[a:] / (1 - math.pow(BETA1, s["step"])), v[a:] / (1 - math.pow(BETA2, s["step"]))
    w[a:] -= LR * (mean / (torch.sqrt(var) + EPS) + case["decay"] * w[a:])
    p = w.clone()
    p[:a] = s["param"][:a].double()
    return [p, w, m, v]
