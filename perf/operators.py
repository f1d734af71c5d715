"""Timed cases of the token-embedding operators: lookup with scaling, its gradient by sorted tokens, the global
gradient norm with clipping, and the update that applies summed gradient rows to the store.

A pass is one call of an operator as a training or serving step makes it (a clipping pass is the norm and the
clipping that uses it, an update pass the update and the read of the rows it wrote).  The plain forms are elementary
torch operations in 32 bits on a table of rows; the framework's calls go through `adapm.ParameterManager`, whose
store holds the same rows.  Outputs are whole: looked-up rows, distinct tokens with their gradient rows and their
number, the norm with every clipped gradient, the updated rows.

Sizes are those of the workloads that the benchmark and the tests name (rows of 64, 200, 300 and 512 floats, 700,000
words, batches of 2^18), and generic ones around them.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
LR, EPS = 0.05, 1e-8


def listed():
    return [
        # --- lookup ------------------------------------------------------------------------------------------
        # one short sequence served alone: latency is everything
        embed("embed_few", vocab=1_400_000, dim=300, batch=1, length=7, ids="int64", out="float32", s=0.0),
        # a training batch: inputs are all but the last token of each sequence (a strided view), ragged ends are
        # padded, rows hold AdaGrad accumulators behind the parameters, the worker holds replicas of its tokens
        embed("embed_batch", vocab=700_000, dim=256, batch=24, length=1023, ids="int64", out="bfloat16", s=1.0,
              adagrad=True, shifted=True, pad=True, held=True),
        # the largest batch over wide rows
        embed("embed_large", vocab=250_000, dim=1024, batch=64, length=4096, ids="int32", out="bfloat16", s=1.0),
        # --- its gradient ------------------------------------------------------------------------------------
        # a few tokens: launches
        grad("grad_few", vocab=1_400_000, dim=300, batch=1, length=37, ids="int32", type="float32", s=0.0),
        # a small batch of 16-bit gradients
        grad("grad_6k", vocab=1_100_000, dim=200, batch=3, length=2003, ids="int64", type="bfloat16", s=1.0),
        # rows of 50 (no vector width divides them evenly), a few hot tokens take most rows, padded ends
        grad("grad_odd", vocab=1_000_003, dim=50, batch=31, length=2113, ids="int64", type="float16", s=1.4, pad=True),
        # the largest batch
        grad("grad_large", vocab=250_000, dim=1024, batch=64, length=4096, ids="int64", type="bfloat16", s=1.0,
             shifted=True),
        # --- norm and clipping -------------------------------------------------------------------------------
        # a small model: launches
        clip("clip_small", tensors=24, total=100_003, types="float32", layout=1),
        # a model of many tensors of every size in both types, packed end to end (odd sizes: unaligned starts),
        # gradients still multiplied by a loss scale
        clip("clip_mixed", tensors=211, total=40_000_003, types="mixed", layout=2, packed=True, loss_scale=1024.0),
        # a few very large ones in 16 bits
        clip("clip_large", tensors=6, total=500_000_000, types="bfloat16", layout=3),
        # --- update ------------------------------------------------------------------------------------------
        # plain SGD on the rows of one small batch, into replicas
        update("update_20k", keys=10_000_000, dim=64, rows=20_011, adagrad=False, held=True),
        # AdaGrad with clipping on the rows of a large batch
        update("update_400k", keys=5_000_000, dim=256, rows=400_003, adagrad=True, held=False),
    ]


def embed(name, vocab, dim, batch, length, ids, out, s, adagrad=False, shifted=False, pad=False, held=False):
    return {"name": name, "kind": "embed", "vocab": vocab, "dim": dim, "batch": batch, "length": length, "ids": ids,
            "type": out, "s": s, "adagrad": adagrad, "shifted": shifted, "pad": pad, "held": held}


def grad(name, vocab, dim, batch, length, ids, type, s, shifted=False, pad=False):
    return {"name": name, "kind": "grad", "vocab": vocab, "dim": dim, "batch": batch, "length": length, "ids": ids,
            "type": type, "s": s, "adagrad": False, "shifted": shifted, "pad": pad, "held": False}


def clip(name, tensors, total, types, layout, packed=False, loss_scale=1.0, clipped=True):
    return {"name": name, "kind": "clip", "tensors": tensors, "total": total, "types": types, "layout": layout,
            "packed": packed, "loss_scale": loss_scale, "clipped": clipped}


def update(name, keys, dim, rows, adagrad, held):
    return {"name": name, "kind": "update", "vocab": keys, "dim": dim, "rows": rows, "adagrad": adagrad, "held": held}


# ---------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed", "grad", "grad", "grad", "clip", "clip", "update", "update"])
    if kind in ("embed", "grad"):
        dim = rng.choice([16, 50, 64, 100, 128, 200, 256, 300, 333, 512, 768, 1000, 1024])
        n = _log(rng, 4, min(1 << 20, (1 << 28) // dim))
        batch = min(n, rng.choice([1, 1, 3, 8, 24, 64]))
        vocab = _log(rng, 1000, min(10_000_000, (1 << 29) // dim))
        ids, type = rng.choice(["int32", "int64"]), rng.choice(["float32", "bfloat16", "float16"])
        s = rng.choice([0.0, 0.8, 1.0, 1.1, 1.4])
        shifted, pad = rng.random() < 0.3, rng.random() < 0.3
        if kind == "grad":
            c = grad("", vocab, dim, batch, n // batch, ids, type, s, shifted, pad)
        else:
            adagrad = dim <= 512 and dim % 4 == 0 and rng.random() < 0.4
            c = embed("", vocab, dim, batch, n // batch, ids, type, s, adagrad, shifted, pad, rng.random() < 0.4)
    elif kind == "clip":
        total = _log(rng, 5_000, 400_000_000)
        tensors = min(_log(rng, 1, 600), total // 16)
        types = rng.choice(["float32", "bfloat16", "float16", "mixed"])
        c = clip("", tensors, total if types != "float32" else max(5_000, total // 2), types, rng.randint(1, 10_000),
                 rng.random() < 0.5, rng.choice([1.0, 1.0, 1024.0]), rng.random() < 0.8)
    else:
        adagrad = rng.random() < 0.6
        dim = rng.choice([16, 64, 100, 128, 200, 256, 300, 512] + ([] if adagrad else [50, 1000]))
        rows = _log(rng, 10, min(1_000_000, 100_000_000 // dim))
        c = update("", max(2 * rows, _log(rng, 1000, (1 << 30) // dim)), dim, rows, adagrad, rng.random() < 0.4)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _ranks(n, size, s, g):
    """n ranks in [0, size), P(rank) falling as (rank + 1)^-s (the bounded power law, rounded down)."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    if s == 0.0:
        x = u * size
    elif s == 1.0:
        x = torch.exp(u * math.log(size + 1.0)) - 1.0
    else:
        x = torch.pow(u * ((size + 1.0) ** (1.0 - s) - 1.0) + 1.0, 1.0 / (1.0 - s)) - 1.0
    return x.to(torch.int64).clamp_(0, size - 1)


def _spread(ranks, size):
    """Ranks to keys by a fixed bijection of [0, size), so that hot keys are not neighbours."""
    a = max(1, int(size * 0.6180339887)) | 1
    while math.gcd(a, size) != 1:
        a += 2
    return (ranks * a + 12345) % size


def _value_len(c):
    return 2 * c["dim"] if c["adagrad"] else -(-c["dim"] // 4) * 4


def _table(c, g):
    """Rows of the store: parameters N(0, 0.1); AdaGrad accumulators as after some training."""
    t = torch.empty((c["vocab"], _value_len(c)), device=DEV)
    if c["adagrad"]:
        t[:, :c["dim"]].normal_(0.0, 0.1, generator=g)
        t[:, c["dim"]:].uniform_(0.05, 1.0, generator=g)
    else:
        t.normal_(0.0, 0.1, generator=g)
    return t


def _tokens(c, g):
    """Sequences of tokens; the ends of the shorter ones hold the padding token 0."""
    B, T = c["batch"], c["length"] + (1 if c["shifted"] else 0)
    t = _spread(_ranks(B * T, c["vocab"], c["s"], g), c["vocab"]).view(B, T)
    if c["pad"]:
        lengths = torch.randint(max(1, T // 2), T + 1, (B, 1), generator=g, device=DEV)
        t = torch.where(torch.arange(T, device=DEV) < lengths, t, torch.zeros_like(t))
    t = t.to(torch.int32 if c["ids"] == "int32" else torch.int64)
    return t[:, :-1] if c["shifted"] else t


def _sizes(c):
    """Element counts and types of a model's tensors, from vectors of a few values to large matrices."""
    rng = random.Random(c["layout"])
    w = [math.exp(rng.uniform(0.0, 6.0)) for _ in range(c["tensors"])]
    sizes = [max(1, int(c["total"] * x / sum(w))) for x in w]
    sizes[sizes.index(max(sizes))] += c["total"] - sum(sizes)
    types = [c["types"] if c["types"] != "mixed" else rng.choice(["float32", "bfloat16"]) for _ in sizes]
    return sizes, types


def _grads(c, g):
    """The model's gradients as views of one buffer per type, and buffers for the clipped ones laid out alike."""
    sizes, types = _sizes(c)
    align = 1 if c["packed"] else 128
    starts, ends = [], {}
    for n, t in zip(sizes, types):
        starts.append(ends.get(t, 0))
        ends[t] = -(-(starts[-1] + n) // align) * align
    flat = {t: torch.zeros(n, dtype=TYPES[t], device=DEV) for t, n in ends.items()}
    outs = {t: torch.zeros_like(f) for t, f in flat.items()}
    views = lambda bufs: [bufs[t][a:a + n] for a, n, t in zip(starts, sizes, types)]   # noqa: E731
    for v in views(flat):
        v.normal_(0.0, 0.01 * c["loss_scale"], generator=g)
    return flat, outs, views(flat), views(outs)


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(1_000_003 * (seed + 1))
    x = {"case": c}
    if c["kind"] == "clip":
        x["flat"], x["out_flat"], x["grads"], x["outs"] = _grads(c, g)
        # a limit well below the usual norm, or one above it
        x["max_norm"] = 0.01 * math.sqrt(c["total"]) * (0.37 if c["clipped"] else 2.0)
        return x
    if c["kind"] == "update":
        # distinct keys, ascending, spread over the store; rows as summed over a batch; the norm that clips them
        step = c["vocab"] // c["rows"]
        x["keys"] = (torch.arange(c["rows"], device=DEV) * step
                     + torch.randint(0, step, (c["rows"],), generator=g, device=DEV)).to(torch.int32)
        x["rows"] = torch.empty((c["rows"], c["dim"]), device=DEV).normal_(0.0, 0.01, generator=g)
        x["norm"] = torch.rand((), generator=g, device=DEV) + 1.5
        x["table"] = _table(c, g)
        return x
    x["tokens"] = _tokens(c, g)
    x["scale"] = math.sqrt(c["dim"])
    if c["kind"] == "embed":
        x["table"] = _table(c, g)
        x["out"] = torch.zeros((c["batch"], c["length"], c["dim"]), dtype=TYPES[c["type"]], device=DEV)
        return x
    n = c["batch"] * c["length"]
    x["grad"] = torch.empty((c["batch"], c["length"], c["dim"]), dtype=TYPES[c["type"]], device=DEV)
    x["grad"].normal_(0.0, 0.01, generator=g)
    # room for as many distinct tokens as there are tokens; what lies behind the last one stays zero
    x["keys"] = torch.empty(n, dtype=torch.int32, device=DEV)
    x["rows"] = torch.zeros((n, c["dim"]), device=DEV)
    x["count"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:
        from paper_2206_00470_gb300 import adapm
        c = case
        if c["kind"] == "clip":
            x["pm"] = adapm.ParameterManager(1, 4, 1, replica_capacity=1)
            x["grads"], x["outs"] = adapm.GradList(x["grads"]), adapm.GradList(x["outs"])
        elif c["kind"] == "grad":
            x["pm"] = adapm.ParameterManager(c["vocab"], _value_len(c), 1, replica_capacity=1)
            x["into"] = adapm.RowGrads(x["keys"], x["rows"], x["count"])
        else:
            touched = x["tokens"] if c["kind"] == "embed" else x["keys"]
            x["pm"] = adapm.ParameterManager(c["vocab"], _value_len(c), 1, init_values=x.pop("table"),
                                             replica_capacity=touched.numel() if c["held"] else 1)
            if c["held"]:
                x["pm"].intent(0, touched, 0, 1 << 40)
    return x


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(x):
    kind = x["case"]["kind"]
    if own:
        return {"embed": _own_embed, "grad": _own_grad, "clip": _own_clip, "update": _own_update}[kind](x)
    return {"embed": _plain_embed, "grad": _plain_grad, "clip": _plain_clip, "update": _plain_update}[kind](x)


def _pad(c):
    return 0 if c["pad"] else None


def _own_embed(x):
    return x["pm"].embed(0, x["tokens"], scale=x["scale"], pad=_pad(x["case"]), out=x["out"])


def _own_grad(x):
    g = x["pm"].embed_grad(0, x["tokens"], x["grad"], scale=x["scale"], pad=_pad(x["case"]), out=x["into"])
    return {"keys": g.keys, "rows": g.rows, "count": g.count}


def _own_clip(x):
    s = 1.0 / x["case"]["loss_scale"]
    norm = x["pm"].grad_norm(x["grads"], scale=s)
    x["pm"].clip_grads(x["grads"], norm, x["max_norm"], scale=s, out=x["outs"])
    return {"norm": norm, "grads": x["out_flat"]}


def _own_update(x):
    c, pm = x["case"], x["pm"]
    pm.push_grads(0, x["keys"], x["rows"], LR, adagrad=c["adagrad"], eps=EPS, norm=x["norm"], max_norm=1.0)
    return pm.pull(0, x["keys"])


def _plain_embed(x):
    c, t = x["case"], x["tokens"].long()
    rows = x["table"][:, :c["dim"]][t] * x["scale"]
    if c["pad"]:
        rows = rows * (t != 0).unsqueeze(-1)
    return rows.to(TYPES[c["type"]])


def _plain_grad(x):
    c, t = x["case"], x["tokens"].reshape(-1).long()
    g = x["grad"].reshape(-1, c["dim"]).float()
    if c["pad"]:
        g, t = g[t != 0], t[t != 0]
    keys, inverse = torch.unique(t, return_inverse=True)
    n, u = c["batch"] * c["length"], keys.numel()
    rows = torch.zeros((n, c["dim"]), device=DEV).index_add_(0, inverse, g * x["scale"])
    padded = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    padded[:u] = keys.to(torch.int32)
    return {"keys": padded, "rows": rows, "count": torch.full((1,), u, dtype=torch.int32, device=DEV)}


def _plain_clip(x):
    s = 1.0 / x["case"]["loss_scale"]
    norm = s * torch.stack([(f.float() * f.float()).sum() for f in x["flat"].values()]).sum().sqrt()
    factor = torch.where(norm <= x["max_norm"], torch.ones_like(norm), x["max_norm"] / norm)
    return {"norm": norm, "grads": {t: (f.float() * (s * factor)).to(f.dtype) for t, f in x["flat"].items()}}


def _plain_update(x):
    c, k = x["case"], x["keys"].long()
    factor = torch.where(x["norm"] <= 1.0, torch.ones_like(x["norm"]), 1.0 / x["norm"])
    g, d, old = x["rows"] * factor, c["dim"], x["table"][k]
    new = old.clone()
    if c["adagrad"]:
        new[:, d:] = old[:, d:] + g * g
        new[:, :d] = old[:, :d] - LR * g / torch.sqrt(old[:, d:] + g * g + EPS)
    else:
        new[:, :d] = old[:, :d] - LR * g
    x["table"][k] = new
    return x["table"][k]


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    x, c = _inputs(case, seed), case
    if c["kind"] == "embed":
        t = x["tokens"].long()
        keep = torch.ones(t.shape, dtype=torch.float64, device=DEV) if not c["pad"] else (t != 0).double()
        return torch.einsum("btd,bt->btd", x["table"].double()[t][..., :c["dim"]], keep * x["scale"])
    if c["kind"] == "grad":
        # sums of the rows of equal tokens as differences of the running sums of the sorted rows
        t = x["tokens"].reshape(-1).long()
        at = torch.argsort(t, stable=True)
        if c["pad"]:
            at = at[t[at] != 0]
        st = t[at]
        last = torch.ones_like(st, dtype=torch.bool)
        last[:-1] = st[1:] != st[:-1]
        sums = x["grad"].reshape(-1, c["dim"])[at].double().cumsum(0)[last]
        sums[1:] -= sums[:-1].clone()
        u, n = sums.shape[0], t.numel()
        rows = torch.zeros((n, c["dim"]), dtype=torch.float64, device=DEV)
        rows[:u] = sums * x["scale"]
        return {"keys": None, "rows": rows, "count": None}
    if c["kind"] == "clip":
        s = 1.0 / c["loss_scale"]
        norm = math.sqrt(sum(float(torch.dot(g.double(), g.double())) for g in x["grads"])) * s
        factor = 1.0 if norm <= x["max_norm"] else x["max_norm"] / norm
        return {"norm": torch.tensor(norm, dtype=torch.float64),
                "grads": {t: f.double() * s * factor for t, f in x["flat"].items()}}
    norm = float(x["norm"])
    g = x["rows"].double() * min(1.0, 1.0 / norm)
    v = x["table"][x["keys"].long()].double()
    if not c["adagrad"]:
        v[:, :c["dim"]] -= LR * g
        return v
    theta, a = v.chunk(2, dim=1)
    a = a + g ** 2
    return torch.cat([theta - LR * g * (a + EPS) ** -0.5, a], dim=1)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def _distinct(n, size, s):
    """Expected number of distinct ranks among n (the bounded power law over [0, size))."""
    r = np.unique(np.round(np.geomspace(1, size + 1, 20_000)).astype(np.int64)).astype(np.float64)
    if s == 0.0:
        cdf = (r - 1.0) / size
    elif s == 1.0:
        cdf = np.log(r) / math.log(size + 1.0)
    else:
        cdf = (r ** (1.0 - s) - 1.0) / ((size + 1.0) ** (1.0 - s) - 1.0)
    ranks = np.diff(r)
    p = np.diff(cdf) / ranks
    return float((ranks * -np.expm1(n * np.log1p(-np.minimum(p, 1.0 - 1e-12)))).sum())


def work(c):
    if c["kind"] == "clip":
        sizes, types = _sizes(c)
        nbytes = sum(n * BYTES[t] for n, t in zip(sizes, types))
        return {"bytes": 2.0 * nbytes + 4, "flops": 3.0 * c["total"]}       # read once, written once
    if c["kind"] == "update":
        rows = c["rows"] * _value_len(c) * 4.0
        grads = c["rows"] * c["dim"] * 4.0
        return {"bytes": c["rows"] * 4.0 + grads + 3.0 * rows,               # rows read, written, returned
                "flops": c["rows"] * c["dim"] * (8.0 if c["adagrad"] else 3.0)}
    n, d, b = c["batch"] * c["length"], c["dim"], BYTES[c["type"]]
    if c["pad"]:   # sequences are three quarters full on average
        n = n * 3 // 4 + 1
    u = _distinct(n, c["vocab"], c["s"])
    ids = c["batch"] * c["length"] * (4.0 if c["ids"] == "int32" else 8.0)
    if c["kind"] == "embed":
        return {"bytes": ids + u * d * 4.0 + c["batch"] * c["length"] * d * b, "flops": n * d * 1.0}
    return {"bytes": ids + n * d * b + u * (4.0 + d * 4.0), "flops": n * d * 1.0 + u * d}
