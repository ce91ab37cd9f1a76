"""Operators of models that keep their parameters in a store: layer norm, a router over experts, orthogonalized updates.

`run` computes them in their plain form (elementary torch operations), or, with `own`, by the framework's calls.  `kind`:

  pull_norm      rows of a batch of keys, normalised: what a model does with the embeddings that it pulls
  norm           layer norm of activations
  norm_grad      its backward pass: the gradients of the input, the weight and the bias
  route          a router over experts as serving calls it: choices, their weights, counts per expert
  route_train    the same with the balance and z losses, and the gradient of the logits
  orthogonalize  Newton-Schulz products on the update of a matrix or of a batch of them, scaled as the store is to add it

Sizes: row lengths and key counts of the workloads in bench.py and of the tests (64, 100, 128, 300, 500, 1000 values), and
generic ones (powers of two, odd sizes) for activations, experts and matrices.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f64": torch.float64, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)    # of the quintic that the orthogonalization iterates
NS_STEPS, NS_EPS, RATE = 5, 1e-7, 0.02
BALANCE, Z = 0.01, 0.001


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # an inference request: the embeddings of a few keys, normalised; nothing but latency
        {"name": "pull_norm_few", "kind": "pull_norm", "keys": 1_000_000, "len": 64, "values": "f32", "out": "f32", "n": 96, "top": 0},
        # a training batch of skewed keys from a large table, the most frequent keys replicated, activations in 16 bits
        {"name": "pull_norm_many", "kind": "pull_norm", "keys": 5_000_000, "len": 128, "values": "f32", "out": "bf16", "n": 1 << 20, "top": 1000},
        # one token of a model that answers: the smallest call
        {"name": "norm_token", "kind": "norm", "n": 1, "len": 4096, "x": "bf16", "w": "bf16"},
        # a long prompt or a training batch
        {"name": "norm_batch", "kind": "norm", "n": 16_384, "len": 4096, "x": "bf16", "w": "f32"},
        # short rows, as embeddings are, in many items; an odd number of them and an odd length
        {"name": "norm_grad_rows", "kind": "norm_grad", "n": 200_003, "len": 101, "x": "f32", "dy": "f32", "w": "f32"},
        # the widest activations of a training step
        {"name": "norm_grad_wide", "kind": "norm_grad", "n": 16_384, "len": 4096, "x": "bf16", "dy": "bf16", "w": "f32"},
        # a few tokens of several requests that are answered together
        {"name": "route_tokens", "kind": "route", "n": 24, "experts": 64, "choose": 2, "type": "bf16", "active": 1.0},
        # a training batch, its padding left out
        {"name": "route_train_batch", "kind": "route_train", "n": 65_536, "experts": 256, "choose": 8, "type": "bf16", "active": 0.9},
        # few experts, float logits, an odd number of tokens
        {"name": "route_train_few", "kind": "route_train", "n": 30_011, "experts": 12, "choose": 1, "type": "f32", "active": 1.0},
        # matrices of relations kept as rows of a store: many small ones
        {"name": "orthogonalize_relations", "kind": "orthogonalize", "batch": 64, "rows": 100, "cols": 100, "type": "f32"},
        # a projection of a model, wider than high, gradients in 16 bits
        {"name": "orthogonalize_wide", "kind": "orthogonalize", "batch": 1, "rows": 1024, "cols": 4096, "type": "bf16"},
        # the largest square matrix, in 32 bits
        {"name": "orthogonalize_large", "kind": "orthogonalize", "batch": 1, "rows": 4096, "cols": 4096, "type": "f32"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm; odd ones as often as even ones."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["pull_norm", "norm", "norm", "norm_grad", "norm_grad", "route", "route_train", "route_train", "orthogonalize", "orthogonalize"])
    if kind == "pull_norm":
        values = rng.choice(["f32", "f32", "f64"])
        length = 4 * _log(rng, 4, 256)
        return {"kind": kind, "keys": _log(rng, 10_000, 640_000_000 // (length * (1 if values == "f32" else 2))), "len": length, "values": values,
                "out": rng.choice(["f32", "bf16", "f16"]) if values == "f32" else "f64",
                "n": _log(rng, 1, min(1 << 20, 100_000_000 // (length * (1 if values == "f32" else 2)))), "top": rng.choice([0, 100, 1000])}
    if kind in ("norm", "norm_grad"):
        x = rng.choice(["f32", "bf16", "bf16", "f16", "f64"])
        length = _log(rng, 8, 16_384)
        c = {"kind": kind, "n": _log(rng, 1, max(1, 60_000_000 // (length * (1 if x != "f64" else 2)))), "len": length, "x": x}
        if kind == "norm_grad":
            c["dy"] = rng.choice(["f32", "bf16", "f16"]) if x == "f32" else x
        c["w"] = x if x in ("f32", "f64") else rng.choice([x, "f32"])
        c["n"] = min(c["n"], 1_000_000)
        return c
    if kind in ("route", "route_train"):
        experts = _log(rng, 4, 512)
        return {"kind": kind, "n": _log(rng, 1, min(1_000_000, 16_000_000 // experts)), "experts": experts, "choose": min(experts, rng.choice([1, 2, 4, 6, 8])),
                "type": rng.choice(["bf16", "f32", "f16"]), "active": rng.choice([1.0, 0.9, 0.5])}
    rows, cols = _log(rng, 8, 4096), _log(rng, 8, 4096)
    return {"kind": kind, "batch": min(_log(rng, 1, 256), max(1, 16_000_000 // (rows * cols))), "rows": rows, "cols": cols, "type": rng.choice(["f32", "bf16", "f16"])}


# ------------------------------------------------------------------------------------------------
# what a user's program has in hand
# ------------------------------------------------------------------------------------------------
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + salt)


def _normal(shape, seed, salt, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, salt), device="cuda").to(dtype)


def _key_of_rank(rank, keys):
    """Ranks spread over the keys, so that frequent keys are not adjacent rows."""
    step = 2_654_435_761 % keys | 1
    while math.gcd(step, keys) != 1:
        step += 2
    return ((rank.long() * step + 12_345) % keys).to(torch.int32)


def _inputs(c, seed):
    """The case's inputs, from the seed alone."""
    k = c["kind"]
    if k == "pull_norm":
        dtype = TYPES[c["values"]]
        rank = torch.rand(c["n"], generator=_gen(seed, 1), device="cuda", dtype=torch.float64).mul_(math.log(c["keys"])).exp_().long() - 1   # near Zipf(1)
        return {"table": torch.randn((c["keys"], c["len"]), generator=_gen(seed, 0), device="cuda", dtype=dtype).mul_(0.1).add_(0.02),
                "keys": _key_of_rank(rank.clamp_(0, c["keys"] - 1), c["keys"]),
                "weight": 1 + 0.1 * _normal(c["len"], seed, 2, dtype), "bias": 0.1 * _normal(c["len"], seed, 3, dtype)}
    if k in ("norm", "norm_grad"):
        x = (_normal((c["n"], c["len"]), seed, 0) * 1.5 + 0.3).to(TYPES[c["x"]])
        w = TYPES[c["w"]]
        st = {"x": x, "weight": (1 + 0.1 * _normal(c["len"], seed, 1)).to(w), "bias": (0.1 * _normal(c["len"], seed, 2)).to(w)}
        if k == "norm_grad":
            st["dy"] = (_normal((c["n"], c["len"]), seed, 3) * 0.01).to(TYPES[c["dy"]])
            # what the forward pass left
            wide = x.double()
            mean = wide.mean(1)
            rstd = (wide.square().mean(1) - mean.square()).clamp_(min=0).add_(EPS).rsqrt()
            keep = torch.float64 if c["x"] == "f64" else torch.float32
            st["mean"], st["rstd"] = mean.to(keep), rstd.to(keep)
        return st
    if k in ("route", "route_train"):
        n, E = c["n"], c["experts"]
        logits = (_normal((n, E), seed, 0) + 0.7 * _normal(E, seed, 1)).to(TYPES[c["type"]])     # some experts are asked for more often
        st = {"logits": logits, "active": None}
        if c["active"] < 1:
            st["active"] = torch.arange(n, device="cuda") % 1024 < 1024 * c["active"]            # sequences of 1024 tokens, padded at their ends
        if k == "route_train":
            st["dweight"] = _normal((n, c["choose"]), seed, 2) * 1e-3
            st["dloss"] = torch.ones((), device="cuda")
        return st
    r, q = c["rows"], c["cols"]
    low = max(1, min(r, q) // 8)                            # a gradient: a part of low rank, and noise
    g = _normal((c["batch"], r, low), seed, 0) @ _normal((c["batch"], low, q), seed, 1) / math.sqrt(low) + 0.3 * _normal((c["batch"], r, q), seed, 2)
    return {"update": (1e-3 * g).to(TYPES[c["type"]])}


def prepare(case, seed):
    st = _inputs(case, int(seed))
    st["case"] = case
    if own:
        from paper_2104_00501_b200 import binding
        if case["kind"] == "pull_norm":
            st["store"] = s = binding.Store(case["keys"], case["len"], sync_interval=0, value_bytes=8 if case["values"] == "f64" else 4)
            s.write_table(0, st.pop("table"))
            top = min(case["top"], case["keys"] // 4)
            if top:
                s.set_management(_key_of_rank(torch.arange(top, device="cuda"), case["keys"]), binding.REPLICATE)
        else:
            st["store"] = binding.Store(64, 64)             # the program's store, whose operators these are
    return st


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(st):
    return globals()[("_own_" if own else "_plain_") + st["case"]["kind"]](st, st["case"])


def _own_pull_norm(st, c):
    y, mean, rstd, rows = st["store"].pull_norm(st["keys"], st["weight"], st["bias"], eps=EPS, out_dtype=TYPES[c["out"]], rows=True)
    return {"y": y, "mean": mean, "rstd": rstd, "rows": rows}


def _own_norm(st, c):
    return st["store"].layer_norm(st["x"], st["weight"], st["bias"], eps=EPS)


def _own_norm_grad(st, c):
    return st["store"].layer_norm_grad(st["x"], st["dy"], st["mean"], st["rstd"], st["weight"])


def _own_route(st, c):
    r = st["store"].route(st["logits"], c["choose"], active=st["active"], renormalize=True)
    return {"choice": r.choice, "weight": r.weight, "counts": r.counts}


def _own_route_train(st, c):
    r = st["store"].route(st["logits"], c["choose"], active=st["active"], balance=BALANCE, z=Z)
    d = st["store"].route_grad(st["logits"], r, dweight=st["dweight"], dloss=st["dloss"])
    return {"choice": r.choice, "weight": r.weight, "counts": r.counts, "tokens": r.tokens, "prob": r.prob, "loss": r.loss, "dlogits": d}


def _own_orthogonalize(st, c):
    return st["store"].orthogonalize(st["update"], steps=NS_STEPS, coefficients=COEFFICIENTS, eps=NS_EPS, scale=_rate(c))


def _rate(c):
    return -RATE * math.sqrt(max(1.0, c["rows"] / c["cols"]))


def _wide(t):
    return t if t.dtype == torch.float64 else t.float()


def _plain_normalised(x, weight, bias, out):
    x = _wide(x)
    mean = x.sum(1) / x.shape[1]
    centred = x - mean[:, None]
    rstd = torch.rsqrt((centred * centred).sum(1) / x.shape[1] + EPS)
    return (centred * rstd[:, None] * _wide(weight) + _wide(bias)).to(out), mean, rstd


def _plain_pull_norm(st, c):
    rows = st["table"][st["keys"].long()]
    y, mean, rstd = _plain_normalised(rows, st["weight"], st["bias"], TYPES[c["out"]])
    return {"y": y, "mean": mean, "rstd": rstd, "rows": rows}


def _plain_norm(st, c):
    return _plain_normalised(st["x"], st["weight"], st["bias"], st["x"].dtype)


def _plain_norm_grad(st, c):
    x, dy, w = _wide(st["x"]), st["dy"].to(torch.float64 if c["x"] == "f64" else torch.float32), _wide(st["weight"])
    hat = (x - st["mean"][:, None]) * st["rstd"][:, None]
    g = dy * w
    a, b = g.sum(1) / c["len"], (g * hat).sum(1) / c["len"]
    dx = (g - a[:, None] - hat * b[:, None]) * st["rstd"][:, None]
    return dx.to(st["x"].dtype), (dy * hat).sum(0).to(st["weight"].dtype), dy.sum(0).to(st["weight"].dtype)


def _plain_choices(st, c):
    x = st["logits"].float()
    n, E, k = c["n"], c["experts"], c["choose"]
    active = torch.ones(n, dtype=torch.bool, device=x.device) if st["active"] is None else st["active"]
    choice = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    choice = torch.where(active[:, None], choice, -1)
    counts = torch.zeros(E + 1, dtype=torch.int64, device=x.device)
    counts = counts.scatter_add_(0, (choice + 1).reshape(-1), torch.ones_like(choice).reshape(-1))[1:]
    return x, active, choice, counts


def _plain_route(st, c):
    x, active, choice, counts = _plain_choices(st, c)
    z = x.gather(1, choice.clamp(min=0))
    e = torch.exp(z - z[:, :1]) * active[:, None]
    return {"choice": choice.to(torch.int32), "weight": e / e.sum(1, keepdim=True).clamp(min=1), "counts": counts}


def _plain_route_train(st, c):
    x, active, choice, counts = _plain_choices(st, c)
    E, k = c["experts"], c["choose"]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    p = torch.where(active[:, None], e / total, 0.0)
    lse = torch.where(active, (top + torch.log(total))[:, 0], 0.0)
    tokens = active.sum()
    T = tokens.clamp(min=1).float()
    at = choice.clamp(min=0)
    weight = p.gather(1, at)
    prob = p.sum(0) / T
    share = counts.float() * (E / k) / T
    balance, z = (share * prob).sum(), (lse * lse).sum() / T
    loss = torch.stack([BALANCE * balance + Z * z, balance, z])
    g = (st["dloss"] * BALANCE * share / T).expand_as(p).scatter_add(1, at, torch.where(active[:, None], st["dweight"], 0.0))
    dlogits = p * (g - (g * p).sum(1, keepdim=True) + (st["dloss"] * Z * 2 * lse / T)[:, None])
    return {"choice": choice.to(torch.int32), "weight": weight, "counts": counts, "tokens": tokens, "prob": prob, "loss": loss,
            "dlogits": dlogits.to(st["logits"].dtype)}


def _plain_orthogonalize(st, c):
    x = st["update"].float()
    tall = c["rows"] > c["cols"]
    if tall:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    a, b, d = COEFFICIENTS
    for _ in range(NS_STEPS):
        g = x @ x.transpose(1, 2)
        x = a * x + (b * g + d * (g @ g)) @ x
    x = _rate(c) * x
    return (x.transpose(1, 2) if tall else x).to(st["update"].dtype).contiguous()


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def _size(name):
    return TYPES[name].itemsize


def work(case):
    c, k = case, case["kind"]
    if k == "pull_norm":
        # near Zipf(1): expected number of distinct keys among n draws whose rank's logarithm is uniform
        n, top, keys, u, lo = c["n"], math.log(c["keys"]), c["keys"], 0.0, 1
        while lo <= keys:
            hi = min(keys + 1, max(lo + 1, int(lo * 1.02)))
            u += (hi - lo) * -math.expm1(-n * (math.log(hi) - math.log(lo)) / (top * (hi - lo)))
            lo = hi
        v = _size(c["values"])
        return {"bytes": n * (4 + c["len"] * (v + _size(c["out"])) + 2 * v) + u * c["len"] * v + 2 * c["len"] * v, "flops": 8 * n * c["len"]}
    if k in ("norm", "norm_grad"):
        n, m, x, w = c["n"], c["len"], _size(c["x"]), _size(c["w"])
        stats = 2 * n * (8 if c["x"] == "f64" else 4)
        if k == "norm":
            return {"bytes": 2 * n * m * x + 2 * m * w + stats, "flops": 8 * n * m}
        return {"bytes": n * m * (2 * x + _size(c["dy"])) + 3 * m * w + stats, "flops": 15 * n * m}
    if k in ("route", "route_train"):
        n, E, t = c["n"], c["experts"], _size(c["type"])
        mask = n if c["active"] < 1 else 0
        if k == "route":
            return {"bytes": n * E * t + mask + 8 * n * c["choose"] + 8 * E, "flops": 6 * n * E}
        return {"bytes": 2 * n * E * t + mask + 12 * n * c["choose"] + 12 * E, "flops": 14 * n * E}
    m, n = sorted((c["rows"], c["cols"]))
    # per step the Gram matrix and its square (symmetric: half of each), and the product with the matrix
    return {"bytes": 2 * c["batch"] * m * n * _size(c["type"]), "flops": c["batch"] * NS_STEPS * (m * m * n + m * m * m + 2 * m * m * n)}


# ------------------------------------------------------------------------------------------------
# the same results in 64 bits, from the definitions
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    c, k = case, case["kind"]
    i = _inputs(c, int(seed))
    if k in ("pull_norm", "norm"):
        x = (torch.index_select(i["table"], 0, i["keys"].to(torch.int64)) if k == "pull_norm" else i["x"]).to(torch.float64)
        rows = x
        var, mean = torch.var_mean(x, dim=-1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = torch.addcmul(i["bias"].to(torch.float64), (x - mean.unsqueeze(-1)) * rstd.unsqueeze(-1), i["weight"].to(torch.float64))
        return {"y": y, "mean": mean, "rstd": rstd, "rows": rows} if k == "pull_norm" else (y, mean, rstd)
    if k == "norm_grad":
        # the Jacobian of x -> (x - mean) rstd, applied to dy * weight; by the statistics that the call is given
        dy, hat, r = i["dy"].double(), (i["x"].double() - i["mean"].double().unsqueeze(1)).mul_(i["rstd"].double().unsqueeze(1)), i["rstd"].double()
        dweight, dbias = torch.einsum("ij,ij->j", dy, hat), dy.sum(0)
        dy *= i["weight"].double()
        along = torch.einsum("ij,ij->i", dy, hat) / c["len"]
        dx = torch.addcmul(dy - dy.mean(1, keepdim=True), hat, along.unsqueeze(1), value=-1).mul_(r.unsqueeze(1))
        return dx, dweight, dbias
    if k in ("route", "route_train"):
        x = i["logits"].double()
        n, E, m = c["n"], c["experts"], c["choose"]
        on = torch.ones(n, dtype=torch.float64, device=x.device) if i["active"] is None else i["active"].double()
        # the larger logit first, the smaller number among equals: one whole-number key per expert would lose bits, so pick one by one
        left, picks = x.clone(), []
        for _ in range(m):
            best = (left == left.amax(1, keepdim=True)).to(torch.uint8).argmax(1)
            picks.append(best)
            left.scatter_(1, best[:, None], -math.inf)
        choice = torch.stack(picks, 1)
        counts = torch.zeros(E, dtype=torch.float64, device=x.device).index_add_(0, choice.reshape(-1), on.repeat_interleave(m))
        kept = torch.where(on[:, None] > 0, choice, -1).to(torch.int32)
        if k == "route":
            return {"choice": kept, "weight": torch.softmax(x.gather(1, choice), 1) * on[:, None], "counts": counts.long()}
        p = torch.softmax(x, 1)
        T = max(1.0, float(on.sum()))
        f, P = counts * E / (m * T), (p * on[:, None]).sum(0) / T
        lse = torch.logsumexp(x, 1)
        balance, z = (f * P).sum(), (on * lse ** 2).sum() / T
        up = torch.zeros_like(p).scatter_(1, choice, i["dweight"].double()) + BALANCE * f / T
        d = p * (up - (up * p).sum(1, keepdim=True)) + (2 * Z / T) * lse[:, None] * p
        return {"choice": kept, "weight": p.gather(1, choice) * on[:, None], "counts": counts.long(), "tokens": on.sum().long(), "prob": P,
                "loss": torch.stack([BALANCE * balance + Z * z, balance, z]), "dlogits": d * on[:, None]}
    # the iteration maps every singular value s to s (a + b s^2 + d s^4) and keeps the singular vectors: out = U diag(product of
    # the factors) U^T X, with U and s^2 from the eigenvalues of X X^T
    g = i["update"].double()
    x = g.transpose(1, 2) if c["rows"] > c["cols"] else g
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + NS_EPS)
    s2, u = torch.linalg.eigh(x @ x.transpose(1, 2))
    a, b, d = COEFFICIENTS
    factor = torch.ones_like(s2)
    for _ in range(NS_STEPS):
        f = a + b * s2 + d * s2 * s2
        factor, s2 = factor * f, s2 * f * f
    x = _rate(c) * ((u * factor.unsqueeze(1)) @ (u.transpose(1, 2) @ x))
    return (x.transpose(1, 2) if c["rows"] > c["cols"] else x).contiguous()
