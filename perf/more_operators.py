"""Timed cases of the dense operators of a token model's step, between the lookup of its embedding and the
embedding's gradient: layer norm and its gradient, matrix products with bias, activation and residual and their
gradients, and the loss that distils a teacher's top logits, with its gradient.

A pass is one call of an operator as a training or serving step makes it.  The plain forms are elementary torch
operations in 32 bits; the framework's calls go through `adapm.ParameterManager`.  Outputs are whole: normalised rows
and their statistics, every gradient, the losses of all rows, products with the values kept for the backward pass.

Sizes are those of the workloads that the benchmark and the tests name (rows of 64, 200, 256 and 300 floats, 250,000
and 700,000 words, sequences of 1023) and generic ones around them.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
ACTIVATIONS = ["none", "relu", "gelu", "gelu_tanh", "silu", "tanh"]
EPS = 1e-5
PAD = -100   # the label of a position behind the end of a sequence


def listed():
    return [
        # --- layer norm ----------------------------------------------------------------------------------------
        # one token of one sequence: latency is everything
        norm("norm_one", batch=1, length=1, dim=4096, type="bfloat16"),
        # a training batch, all but the last token of each sequence (a strided view), parameters in 32 bits
        norm("norm_batch", batch=64, length=1023, dim=1024, type="bfloat16", shifted=True),
        # its gradient for rows that no vector width divides
        norm("norm_grad_odd", batch=5, length=1021, dim=1001, type="float16", grad=True),
        # the gradient of the largest batch
        norm("norm_grad_large", batch=64, length=4096, dim=1024, type="bfloat16", grad=True),
        # --- products ------------------------------------------------------------------------------------------
        # one token through one layer: the weights are what has to be read
        linear("linear_one", rows=1, ins=4096, outs=4096, type="bfloat16", act="silu", bias=True),
        # sizes that nothing divides, output as logits in 32 bits
        linear("linear_odd", rows=1021, ins=333, outs=5003, type="float16", act="none", bias=True, out="float32"),
        # a training batch through a wide layer, with what its backward pass needs
        linear("linear_large", rows=8192, ins=4096, outs=8192, type="bfloat16", act="gelu_tanh", bias=True, keep=True,
               residual=True),
        # gradients of a small layer with weights stored by output
        linear("linear_grad_small", rows=777, ins=256, outs=1000, type="float16", act="tanh", bias=True, by_out=True,
               grad=True),
        # gradients of the wide layer
        linear("linear_grad_large", rows=8192, ins=4096, outs=4096, type="bfloat16", act="gelu_tanh", bias=True,
               grad=True),
        # --- distillation --------------------------------------------------------------------------------------
        # a few tokens: launches
        distill("distill_few", batch=1, length=7, vocab=32_000, top=16, type="float32", temperature=1.0),
        # odd vocabulary, padded sequences, labels beside the teacher, a softened teacher
        distill("distill_odd", batch=3, length=1021, vocab=50_021, top=20, type="bfloat16", temperature=2.0,
                labels=True, pad=True, shifted=True),
        # the largest vocabulary and batch
        distill("distill_large", batch=4, length=1024, vocab=250_000, top=64, type="bfloat16", temperature=1.0,
                labels=True),
    ]


def norm(name, batch, length, dim, type, shifted=False, grad=False, params="float32"):
    return {"name": name, "kind": "norm_grad" if grad else "norm", "batch": batch, "length": length, "dim": dim,
            "type": type, "shifted": shifted, "params": params}


def linear(name, rows, ins, outs, type, act, bias=False, residual=False, keep=False, by_out=False, out=None, wide=0,
           grad=False):
    return {"name": name, "kind": "linear_grad" if grad else "linear", "rows": rows, "ins": ins, "outs": outs,
            "type": type, "act": act, "bias": bias, "residual": residual, "keep": keep, "by_out": by_out,
            "out": out or type, "wide": wide}


def distill(name, batch, length, vocab, top, type, temperature, labels=False, pad=False, shifted=False, grad=True):
    return {"name": name, "kind": "distill", "batch": batch, "length": length, "vocab": vocab, "top": top,
            "type": type, "temperature": temperature, "labels": labels, "pad": pad, "shifted": shifted, "grad": grad}


# ---------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "norm_grad", "linear", "linear", "linear_grad", "distill", "distill"])
    type = rng.choice(["float32", "bfloat16", "float16"])
    if kind in ("norm", "norm_grad"):
        # rows of one element to rows that no block holds in its registers
        dim = _log(rng, 1, 40_000) if rng.random() < 0.5 else rng.choice([64, 200, 256, 300, 512, 1024, 2048, 4096, 8192])
        n = _log(rng, 1, min(1 << 20, (1 << 27) // dim))
        batch = min(n, rng.choice([1, 1, 3, 8, 64]))
        c = norm("", batch, max(1, n // batch), dim, type, rng.random() < 0.3, kind == "norm_grad",
                 rng.choice(["float32", "float32", type]))
    elif kind in ("linear", "linear_grad"):
        type = rng.choice(["bfloat16", "float16"])
        size = lambda: _log(rng, 16, 8192) if rng.random() < 0.5 else rng.choice([64, 200, 256, 300, 512, 1024, 2048, 4096])   # noqa: E731
        ins, outs = size(), size()
        rows = _log(rng, 1, min(16_384, (1 << 37) // (ins * outs)))
        grad = kind == "linear_grad"
        c = linear("", rows, ins, outs, type, rng.choice(ACTIVATIONS), rng.random() < 0.7,
                   not grad and rng.random() < 0.4, not grad and rng.random() < 0.4, rng.random() < 0.4,
                   rng.choice([type, type, "float32"]), rng.choice([0, 0, 8, 5]), grad)
    else:
        vocab = _log(rng, 50, 250_000) if rng.random() < 0.7 else rng.choice([700_000, 32_000, 65_536])
        n = _log(rng, 1, min(1 << 16, (1 << 28) // vocab))
        batch = min(n, rng.choice([1, 1, 3, 8]))
        c = distill("", batch, max(1, n // batch), vocab, min(vocab, _log(rng, 1, 256)), type,
                    rng.choice([1.0, 1.0, 2.0, 4.0, 0.7]), rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.3,
                    rng.random() < 0.7)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(g, shape, type, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=TYPES[type], device=DEV).normal_(mean, std, generator=g)


def _seen(x, c):
    """The batch without the last position of each sequence, as a next-token model takes it, or the whole of it."""
    return x[:, :-1] if c["shifted"] else x


def _norm_inputs(c, g):
    shape = (c["batch"], c["length"] + (1 if c["shifted"] else 0), c["dim"])
    x = {"x": _seen(_normal(g, shape, c["type"], 1.5, 0.3), c)}
    x["weight"] = _normal(g, (c["dim"],), c["params"], 0.2, 1.0)
    x["bias"] = _normal(g, (c["dim"],), c["params"], 0.2)
    rows = (c["batch"], c["length"])
    if c["kind"] == "norm":
        x["out"] = torch.zeros((*rows, c["dim"]), dtype=TYPES[c["type"]], device=DEV)
        x["stats"] = torch.zeros((*rows, 2), device=DEV)
        return x
    x["grad"] = _normal(g, (*rows, c["dim"]), c["type"], 0.1)
    # (in parts, so that the forward pass of a large batch takes little room)
    f = x["x"].double() if c["dim"] * c["batch"] * c["length"] < 1 << 20 else x["x"].float()
    mean = f.mean(-1)
    x["stats"] = torch.stack([mean.float(), ((f - mean.unsqueeze(-1)).square().mean(-1) + EPS).rsqrt().float()], -1)
    x["dx"] = torch.zeros((*rows, c["dim"]), dtype=TYPES[c["type"]], device=DEV)
    x["dweight"], x["dbias"] = torch.zeros_like(x["weight"]), torch.zeros_like(x["bias"])
    return x


def _linear_inputs(c, g):
    m, k, n, t = c["rows"], c["ins"], c["outs"], c["type"]
    x = {"x": _normal(g, (m, k + c["wide"]), t)[:, :k]}   # (wide: the columns of a wider buffer)
    w = _normal(g, (n, k) if c["by_out"] else (k, n), t, 1.0 / math.sqrt(k))
    x["weight"] = w.t() if c["by_out"] else w
    x["bias"] = _normal(g, (n,), t, 0.2) if c["bias"] else None
    if c["kind"] == "linear":
        x["residual"] = _normal(g, (m, n), c["out"]) if c["residual"] else None
        x["out"] = torch.zeros((m, n), dtype=TYPES[c["out"]], device=DEV)
        x["pre"] = torch.zeros((m, n), dtype=TYPES[t], device=DEV) if c["keep"] else None
        return x
    x["grad"] = _normal(g, (m, n), t, 0.1)
    x["pre"] = _normal(g, (m, n), t) if c["act"] != "none" else None
    x["dx"] = torch.zeros((m, k), dtype=TYPES[t], device=DEV)
    x["dweight"] = torch.zeros_like(w).t() if c["by_out"] else torch.zeros_like(w)
    x["dbias"] = torch.zeros(n, dtype=TYPES[t], device=DEV) if c["bias"] else None
    return x


def _distill_inputs(c, g):
    B, T, V, top = c["batch"], c["length"], c["vocab"], c["top"]
    logits = _normal(g, (B, T + (1 if c["shifted"] else 0), V), c["type"], 2.0)
    x = {"logits": _seen(logits, c)}
    # distinct ids per row: a random start, then random gaps
    gaps = torch.randint(1, max(1, V // top) + 1, (B, T, top), generator=g, device=DEV)
    ids = (gaps.cumsum(-1) + torch.randint(0, V, (B, T, 1), generator=g, device=DEV)) % V
    teacher = (torch.empty((B, T, top), device=DEV).normal_(4.0, 2.0, generator=g)).sort(-1, descending=True)[0]
    teacher = teacher.to(TYPES[c["type"]])
    # the student half agrees
    x["logits"].scatter_(-1, ids, (0.5 * teacher.float()
                                   + torch.empty((B, T, top), device=DEV).normal_(0.0, 1.0, generator=g)).to(logits.dtype))
    labels = torch.where(torch.rand((B, T), generator=g, device=DEV) < 0.7, ids[..., 0],
                         torch.randint(0, V, (B, T), generator=g, device=DEV))
    # some lists are shorter (their ends hold -1), and positions behind the end of a sequence have none
    kept = torch.randint(1, 4 * top + 1, (B, T, 1), generator=g, device=DEV)
    if c["pad"]:
        lengths = torch.randint(max(1, T // 2), T + 1, (B, 1), generator=g, device=DEV)
        behind = torch.arange(T, device=DEV) >= lengths
        labels = labels.masked_fill(behind, PAD)
        kept = kept.masked_fill(behind.unsqueeze(-1), 0)
    x["ids"] = ids.masked_fill(torch.arange(top, device=DEV) >= kept, -1)
    x["teacher"] = teacher
    x["labels"] = labels if c["labels"] else None
    x["soft"], x["hard"] = (0.7, 0.3) if c["labels"] else (1.0, 0.0)
    # the mean over all positions; 16-bit gradients of the narrow range are multiplied by a loss scale
    x["scale"] = (1024.0 if c["type"] == "float16" else 1.0) / (B * T)
    x["loss"] = torch.zeros((B, T), device=DEV)
    x["grad"] = torch.zeros((B, T, V), dtype=TYPES[c["type"]], device=DEV) if c["grad"] else None
    return x


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(1_000_003 * (seed + 1))
    if c["kind"] in ("norm", "norm_grad"):
        x = _norm_inputs(c, g)
    elif c["kind"] in ("linear", "linear_grad"):
        x = _linear_inputs(c, g)
    else:
        x = _distill_inputs(c, g)
    x["case"] = c
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:
        from paper_2206_00470_gb300 import adapm
        x["pm"] = adapm.ParameterManager(1, 4, 1, replica_capacity=1)
        if case["kind"] == "norm_grad":
            x["into"] = adapm.NormGrads(x["dx"], x["dweight"], x["dbias"])
        elif case["kind"] == "linear_grad":
            x["into"] = adapm.LinearGrads(x["dx"], x["dweight"], x["dbias"])
    return x


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(x):
    kind = x["case"]["kind"]
    if own:
        return {"norm": _own_norm, "norm_grad": _own_norm_grad, "linear": _own_linear, "linear_grad": _own_linear_grad,
                "distill": _own_distill}[kind](x)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "linear": _plain_linear,
            "linear_grad": _plain_linear_grad, "distill": _plain_distill}[kind](x)


def _own_norm(x):
    out = x["pm"].layer_norm(x["x"], x["weight"], x["bias"], eps=EPS, out=x["out"], stats=x["stats"])
    return {"out": out, "stats": x["stats"]}


def _own_norm_grad(x):
    d = x["pm"].layer_norm_grad(x["x"], x["grad"], x["stats"], x["weight"], out=x["into"])
    return {"x": d.x, "weight": d.weight, "bias": d.bias}


def _own_linear(x):
    out = x["pm"].linear(x["x"], x["weight"], x["bias"], activation=x["case"]["act"], residual=x["residual"],
                         out=x["out"], pre=x["pre"])
    return {"out": out, "pre": x["pre"]} if x["case"]["keep"] else {"out": out}


def _own_linear_grad(x):
    d = x["pm"].linear_grad(x["x"], x["weight"], x["grad"], pre=x["pre"], activation=x["case"]["act"], out=x["into"])
    out = {"x": d.x, "weight": d.weight}
    return {**out, "bias": d.bias} if x["case"]["bias"] else out


def _own_distill(x):
    loss = x["pm"].distill(x["logits"], x["ids"], x["teacher"], temperature=x["case"]["temperature"], soft=x["soft"],
                           labels=x["labels"], hard=x["hard"], pad=PAD, scale=x["scale"], grad=x["grad"], loss=x["loss"])
    return {"loss": loss, "grad": x["grad"]} if x["case"]["grad"] else {"loss": loss}


def _plain_norm(x):
    f = x["x"].float()
    mean = f.mean(-1, keepdim=True)
    f = f - mean
    r = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    y = f * r * x["weight"].float() + x["bias"].float()
    return {"out": y.to(x["x"].dtype), "stats": torch.cat([mean, r], -1)}


def _plain_norm_grad(x):
    mean, r = x["stats"].unsqueeze(-2).unbind(-1)
    h = (x["x"].float() - mean) * r
    dy = x["grad"].float()
    g = dy * x["weight"].float()
    dx = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    return {"x": dx.to(x["x"].dtype), "weight": (dy * h).sum((0, 1)).to(x["weight"].dtype),
            "bias": dy.sum((0, 1)).to(x["bias"].dtype)}


def _act(z, name):
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return torch.tanh(z) if name == "tanh" else z


def _slope(z, name):
    if name == "relu":
        return (z > 0.0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return 1.0 - torch.tanh(z) ** 2


def _plain_linear(x):
    z = x["x"].float() @ x["weight"].float()
    if x["bias"] is not None:
        z = z + x["bias"].float()
    y = _act(z, x["case"]["act"])
    if x["residual"] is not None:
        y = y + x["residual"].float()
    out = {"out": y.to(TYPES[x["case"]["out"]])}
    return {**out, "pre": z.to(x["x"].dtype)} if x["case"]["keep"] else out


def _plain_linear_grad(x):
    dz = x["grad"].float()
    if x["pre"] is not None:
        dz = dz * _slope(x["pre"].float(), x["case"]["act"])
    t = x["x"].dtype
    dweight = dz.t() @ x["x"].float() if x["case"]["by_out"] else x["x"].float().t() @ dz
    out = {"x": (dz @ x["weight"].float().t()).to(t), "weight": (dweight.t() if x["case"]["by_out"] else dweight).to(t)}
    return {**out, "bias": dz.sum(0).to(t)} if x["case"]["bias"] else out


def _plain_distill(x):
    c, T = x["case"], x["case"]["temperature"]
    s = x["logits"].float()
    here = x["ids"] >= 0
    at = x["ids"].clamp(min=0)
    some = here.any(-1, keepdim=True)
    t = torch.where(here, x["teacher"].float() / T, torch.full_like(x["teacher"], -1e30, dtype=torch.float32))
    p = torch.exp(t - t.amax(-1, keepdim=True)) * here
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    top = s.amax(-1, keepdim=True)
    e = torch.exp((s - top) / T)
    total = e.sum(-1, keepdim=True)
    log_q = (s.gather(-1, at) - top) / T - torch.log(total)
    loss = x["soft"] * T * T * (p * (torch.where(p > 0, torch.log(p.clamp(min=1e-38)), p) - log_q)).sum(-1)
    if c["grad"]:
        d = e.mul_(x["soft"] * T * some / total)
        d.scatter_add_(-1, at, -x["soft"] * T * p)
    del e
    if x["labels"] is not None:
        marked = (x["labels"] != PAD).unsqueeze(-1)
        label = x["labels"].clamp(min=0).unsqueeze(-1)
        e = torch.exp(s - top)
        total = e.sum(-1, keepdim=True)
        loss = loss - x["hard"] * ((s.gather(-1, label) - top - torch.log(total)) * marked).squeeze(-1)
        if c["grad"]:
            d.add_(e.mul_(x["hard"] * marked / total))
            d.scatter_add_(-1, label, -x["hard"] * marked.float())
    return {"loss": loss, "grad": d.mul_(x["scale"]).to(x["logits"].dtype)} if c["grad"] else {"loss": loss}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    x, c = _inputs(case, seed), case
    f = {k: v.double() for k, v in x.items()
         if isinstance(v, torch.Tensor) and k in ("x", "weight", "bias", "grad", "stats", "residual", "pre")
         and c["kind"] != "distill"}
    if c["kind"] == "norm":
        var, mean = torch.var_mean(f["x"], -1, correction=0, keepdim=True)
        r = (var + EPS) ** -0.5
        return {"out": torch.addcmul(f["bias"], (f["x"] - mean) * r, f["weight"]), "stats": torch.cat([mean, r], -1)}
    if c["kind"] == "norm_grad":
        n, r = c["dim"], f["stats"][..., 1:]
        h = (f["x"] - f["stats"][..., :1]).mul_(r)
        g = f["grad"] * f["weight"]
        dx = (g - (g.sum(-1, keepdim=True) + h * (g * h).sum(-1, keepdim=True)) / n).mul_(r)
        return {"x": dx, "weight": torch.einsum("btd,btd->d", f["grad"], h), "bias": torch.einsum("btd->d", f["grad"])}
    if c["kind"] == "linear":
        z = f["x"] @ f["weight"]
        z = z + f["bias"] if "bias" in f else z
        y = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
             "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh"), "tanh": torch.tanh}[c["act"]](z)
        y = y + f["residual"] if "residual" in f else y
        return {"out": y, "pre": z} if c["keep"] else {"out": y}
    if c["kind"] == "linear_grad":
        dz = f["grad"] * _slope(f["pre"], c["act"]) if "pre" in f else f["grad"]
        out = {"x": dz @ f["weight"].mT, "weight": torch.einsum("mk,mn->kn", f["x"], dz)}
        return {**out, "bias": dz.sum(0)} if c["bias"] else out
    # distillation: log-softmax of the student at both temperatures, dense teacher probabilities
    T, V, rows = c["temperature"], c["vocab"], c["batch"] * c["length"]
    ids, teacher = x["ids"].reshape(rows, -1), x["teacher"].reshape(rows, -1).double()
    loss = torch.zeros(rows, dtype=torch.float64, device=DEV)
    grad = torch.zeros((rows, V), dtype=torch.float64, device=DEV) if c["grad"] else None
    step = max(1, (1 << 27) // V)
    for a in range(0, rows, step):
        b, t = min(rows, a + step), c["length"]
        at = torch.arange(a, b, device=DEV)
        s = x["logits"][at // t, at % t].double()
        here = ids[a:b] >= 0
        p = torch.nan_to_num(torch.softmax((teacher[a:b] / T).masked_fill(~here, -math.inf), -1))
        dense = torch.zeros_like(s).scatter_add_(-1, ids[a:b].clamp(min=0), p)
        log_q = torch.log_softmax(s / T, -1)
        loss[a:b] = x["soft"] * T ** 2 * (torch.xlogy(p, p).sum(-1) - (dense * log_q).sum(-1))
        d = x["soft"] * T * (log_q.exp() * here.any(-1, keepdim=True) - dense)
        if x["labels"] is not None:
            label = x["labels"].reshape(rows)[a:b]
            marked = label != PAD
            log_c = torch.log_softmax(s, -1)
            one = torch.zeros_like(s).scatter_(-1, label.clamp(min=0).unsqueeze(-1), 1.0) * marked.unsqueeze(-1)
            loss[a:b] -= x["hard"] * (one * log_c).sum(-1)
            d += x["hard"] * (log_c.exp() * marked.unsqueeze(-1) - one)
        if c["grad"]:
            grad[a:b] = d * x["scale"]
    shape = (c["batch"], c["length"])
    return {"loss": loss.view(shape), "grad": grad.view(*shape, V)} if c["grad"] else {"loss": loss.view(shape)}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    b = BYTES[c["type"]]
    if c["kind"] in ("norm", "norm_grad"):
        n, p = c["batch"] * c["length"], BYTES[c["params"]]
        if c["kind"] == "norm":   # rows read and written, statistics written
            return {"bytes": n * (2.0 * c["dim"] * b + 8) + 2.0 * c["dim"] * p, "flops": n * c["dim"] * 7.0}
        return {"bytes": n * (3.0 * c["dim"] * b + 8) + 3.0 * c["dim"] * p, "flops": n * c["dim"] * 14.0}
    if c["kind"] in ("linear", "linear_grad"):
        m, k, n = c["rows"], c["ins"], c["outs"]
        if c["kind"] == "linear":
            outs = BYTES[c["out"]] * (2.0 if c["residual"] else 1.0) + (b if c["keep"] else 0)
            return {"bytes": (m * k + k * n + (n if c["bias"] else 0)) * b + m * n * outs, "flops": 2.0 * m * k * n}
        reads = m * n * (1.0 if c["act"] == "none" else 2.0)
        return {"bytes": (2.0 * (m * k + k * n) + reads + (n if c["bias"] else 0)) * b, "flops": 4.0 * m * k * n}
    n = c["batch"] * c["length"]
    read = n * 0.75 + 1 if c["pad"] else n   # sequences are three quarters full on average
    lists = n * c["top"] * (8.0 + b) + n * (12.0 if c["labels"] else 4.0)
    return {"bytes": lists + c["vocab"] * b * (read + (n if c["grad"] else 0)),
            "flops": read * c["vocab"] * (8.0 if c["grad"] else 4.0) * (2 if c["labels"] else 1)}
