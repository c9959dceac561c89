"""Performance cases of what serves a split model next to its reductions with
fewer bytes: a layer of experts for a few tokens (``experts``: router, choice,
the chosen experts' gated products and their weighted sum), a matrix product of
8-bit integers with a scale for each token and each channel (``linear8``), and
the rounding of rows to such integers (``quantise``).

A case names the operator (``op``), its sizes and types, and how the data lies:
``slack`` elements more lie between the rows of x than they are long (a slice
of a wider array).  ``experts``: ``total`` experts of which this rank holds
``local`` from number ``first`` on, ``top`` chosen for each token, their shares
adding up to one where ``normalise``; ``weights`` is the type that the experts
are held in, "int8" with a scale for each of their channels.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}
SIZES = {"bfloat16": 2, "float16": 2, "float32": 4, "int8": 1}


def _quantise(name, rows, n, dtype, slack=0):
    return {"name": name, "op": "quantise", "rows": rows, "n": n, "dtype": dtype, "slack": slack}


def _linear8(name, rows, n_in, n_out, out="bfloat16", bias=False, residual=False, slack=0):
    return {"name": name, "op": "linear8", "rows": rows, "n_in": n_in, "n_out": n_out, "out": out,
            "bias": bias, "residual": residual, "slack": slack}


def _experts(name, rows, n_model, n_hidden, total, top, dtype="bfloat16", weights=None, out=None,
             act="silu", first=0, local=None, normalise=True, slack=0):
    return {"name": name, "op": "experts", "rows": rows, "n_model": n_model, "n_hidden": n_hidden,
            "total": total, "top": top, "dtype": dtype, "weights": weights or dtype,
            "out": out or dtype, "act": act, "first": first,
            "local": total - first if local is None else local, "normalise": normalise,
            "slack": slack}


def listed():
    return [
        # the activations of one token of one sequence being answered
        _quantise("quantise_token", 1, 4096, "bfloat16"),
        # a long prompt's, as the float32 sums that a reduction leaves
        _quantise("quantise_sums", 8192, 8192, "float32"),
        # one token, the residual stream added
        _linear8("linear8_token", 1, 4096, 4096, residual=True),
        # a small batch of sequences being answered: one rank's share of a
        # row-parallel product, as the float32 partial that ranks add up
        _linear8("linear8_partial_48_rows", 48, 5120, 2048, out="float32"),
        # a short prompt through odd sizes
        _linear8("linear8_ragged", 333, 2500, 1000, "float16", bias=True, slack=7),
        # a batch of short prompts
        _linear8("linear8_prompt_256", 256, 4096, 4096),
        # a long prompt or a large batch
        _linear8("linear8_prompt", 8192, 4096, 8192, bias=True, residual=True),
        # one token through a few large experts, one rank's eighth of each
        _experts("experts_token", 1, 4096, 1792, 8, 2),
        # a small batch through many small experts
        _experts("experts_8_rows", 8, 2048, 1024, 64, 8, normalise=False),
        # the same experts held in 8-bit integers
        _experts("experts_int8", 16, 2048, 1024, 64, 8, weights="int8"),
        # one rank's eighth of the experts, as the float32 partial that ranks
        # add up; many tokens choose none of them
        _experts("experts_share", 24, 4096, 1000, 128, 4, "float16", out="float32", act="gelu_tanh",
                 first=32, local=16),
        # as many tokens as the layer takes, nearly every expert chosen
        _experts("experts_64_rows", 64, 2048, 1024, 128, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantise", "linear8", "linear8", "experts", "experts", "experts"])
    slack = rng.choice([0, 0, 0, 8, 11])
    even = rng.random() < 0.6   # sizes as models have them: multiples of 64; else as drawn

    def size(lo, hi):
        n = _log(rng, lo, hi)
        return max(64, n // 64 * 64) if even else n

    if op == "quantise":
        c = _quantise("", _log(rng, 1, 8192), size(64, 8192),
                      rng.choice(["bfloat16", "float16", "float32"]), slack)
    elif op == "linear8":
        c = _linear8("", _log(rng, 1, 8192), size(64, 8192), size(64, 8192),
                     rng.choice(["bfloat16", "bfloat16", "float16", "float32"]),
                     rng.random() < 0.4, rng.random() < 0.4, slack)
        while work(c)["flops"] > 5.4e11:
            c["rows"] //= 2
    else:
        total = rng.choice([4, 8, 16, 32, 60, 64, 128])
        local = total if rng.random() < 0.6 else max(1, total // rng.choice([2, 4]))
        dtype = rng.choice(["bfloat16", "bfloat16", "float16"])
        c = _experts("", _log(rng, 1, 64), size(128, 4096), size(64, 2048), total,
                     min(total, rng.choice([1, 2, 2, 4, 6, 8])), dtype,
                     rng.choice([dtype, dtype, "int8"]), rng.choice([dtype, dtype, "float32"]),
                     rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]),
                     rng.randrange(total - local + 1), local, rng.random() < 0.7, slack)
        while c["local"] * c["n_model"] * c["n_hidden"] > 128 * 2048 * 1024:
            c["n_hidden"] //= 2
    del c["name"]
    return c


# ------------------------------------------------------------- the inputs

def _normal(g, shape, dtype, scale=1.0):
    return torch.empty(shape, dtype=DTYPES[dtype], device="cuda").normal_(0.0, scale, generator=g)


def _sliced(make, rows, n, slack):
    return make((rows, n + slack))[:, :n]


def _bytes(g, shape):
    """8-bit integers as rounding leaves them: normal values, the largest of a
    row of some thousand at 127."""
    v = torch.empty(shape, dtype=torch.float16, device="cuda").normal_(0.0, 33.0, generator=g)
    return v.round_().clamp_(-127, 127).to(torch.int8)


def _scales(g, shape, typical):
    """Scales of one size, no two alike."""
    return torch.empty(shape, device="cuda").uniform_(0.5, 1.5, generator=g).mul_(typical)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    new = lambda shape, d: torch.empty(shape, dtype=d, device="cuda")  # noqa: E731
    s = {"case": case}
    if own:
        import paper_2109_12626_gb300 as pkg
        s["pkg"] = pkg
    m = case["rows"]
    if case["op"] == "quantise":
        # a few channels are far larger than the others, as activations have them
        n = case["n"]
        x = _sliced(lambda sh: _normal(g, sh, case["dtype"]), m, n, case["slack"])
        far = torch.randint(0, n, (max(1, n // 256),), device="cuda", generator=g)
        x[:, far] *= 8
        s.update(x=x, q=new((m, n), torch.int8), scale=new((m,), torch.float32))
    elif case["op"] == "linear8":
        k, n, out = case["n_in"], case["n_out"], case["out"]
        s["x"] = _sliced(lambda sh: _bytes(g, sh), m, k, case["slack"])
        s["x_scale"] = _scales(g, (m,), 0.03)
        s["w"] = _bytes(g, (n, k))
        s["w_scale"] = _scales(g, (n,), 0.03 * k ** -0.5)
        s["bias"] = _normal(g, (n,), "float32", 0.1) if case["bias"] else None
        s["residual"] = _normal(g, (m, n), out) if case["residual"] else None
        s["y"] = new((m, n), DTYPES[out])
        if own:
            s["plan"] = pkg.Linear8(m, k, n, out=out)
    else:
        d, h, total, local = case["n_model"], case["n_hidden"], case["total"], case["local"]
        dt = case["dtype"]
        s["x"] = _sliced(lambda sh: _normal(g, sh, dt), m, d, case["slack"])
        s["router"] = _normal(g, (total, d), dt, d ** -0.5)
        shapes = {"gate": (local, h, d), "up": (local, h, d), "down": (local, d, h)}
        for name, shape in shapes.items():
            if case["weights"] == "int8":
                s[name] = _bytes(g, shape)
                s[name + "_scale"] = _scales(g, shape[:2], 0.03 * shape[2] ** -0.5)
            else:
                s[name] = _normal(g, shape, dt, shape[2] ** -0.5)
                s[name + "_scale"] = None
        s["y"] = new((m, d), DTYPES[case["out"]])
        s["chosen"] = new((m, case["top"]), torch.int32)
        s["share"] = new((m, case["top"]), torch.float32)
        if own:
            s["plan"] = pkg.Experts(m, d, h, total, case["top"], dt, out=case["out"],
                                    weights=case["weights"], act=case["act"], first=case["first"],
                                    local=local, normalise=case["normalise"])
    return s


# ------------------------------------------------------- the plain form

def _act(name, z):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z))


def _plain_quantise(s):
    # in 64 bits, since 32 would round some values next to a half to the other side
    x = s["x"].double()
    most = x.abs().amax(dim=1, keepdim=True)
    q = torch.round(x * 127 / torch.where(most > 0, most, torch.ones_like(most)))
    return {"q": q.to(torch.int8), "scale": (most / 127).float()[:, 0]}


def _plain_linear8(s):
    # sums of 512 products of 8-bit integers are whole numbers below 2^24, exact in
    # 32 bits; their total may pass 2^24 and is held in 64
    x, w = s["x"].float(), s["w"].float()
    y = None
    for k in range(0, x.shape[1], 512):
        part = (x[:, k:k + 512] @ w[:, k:k + 512].t()).double()
        y = part if y is None else y + part
    y = y.float() * (s["x_scale"][:, None] * s["w_scale"][None, :])
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(DTYPES[s["case"]["out"]])}


def _plain_experts(s):
    case = s["case"]
    x = s["x"].float()
    # the choice is a comparison of values that may lie next to each other: in 64 bits
    logits = s["x"].double() @ s["router"].double().t()
    top, chosen = torch.sort(logits, dim=1, descending=True, stable=True)
    top, chosen = top[:, :case["top"]].float(), chosen[:, :case["top"]]
    logits = logits.float()
    high = top[:, :1]
    share = torch.exp(top - high)
    share = share / (share if case["normalise"] else torch.exp(logits - high)).sum(1, keepdim=True)
    weight = torch.zeros_like(logits).scatter(1, chosen, share)
    y = torch.zeros_like(x)

    def product(a, name, e):
        z = a @ s[name][e].float().t()
        return z if s[name + "_scale"] is None else z * s[name + "_scale"][e]

    for e in range(case["local"]):
        h = _act(case["act"], product(x, "gate", e)) * product(x, "up", e)
        y = y + weight[:, case["first"] + e, None] * product(h, "down", e)
    return {"y": y.to(DTYPES[case["out"]]), "chosen": chosen.to(torch.int32), "share": share}


# ----------------------------------------------------- the framework's calls

def _own_quantise(s):
    s["pkg"].quantise(s["x"], s["q"], s["scale"])
    return {"q": s["q"], "scale": s["scale"]}


def _own_linear8(s):
    s["plan"].forward(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"], bias=s["bias"],
                      residual=s["residual"])
    return {"y": s["y"]}


def _own_experts(s):
    s["plan"].forward(s["x"], s["router"], s["gate"], s["up"], s["down"], s["y"],
                      gate_scale=s["gate_scale"], up_scale=s["up_scale"],
                      down_scale=s["down_scale"], chosen=s["chosen"], share=s["share"])
    return {"y": s["y"], "chosen": s["chosen"], "share": s["share"]}


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# --------------------------------------------------------------- its work

def work(case):
    m = case["rows"]
    if case["op"] == "quantise":
        n = case["n"]
        return {"bytes": m * n * (SIZES[case["dtype"]] + 1) + 4 * m, "flops": 3 * m * n}
    if case["op"] == "linear8":
        k, n, q = case["n_in"], case["n_out"], SIZES[case["out"]]
        return {"bytes": m * k + n * k + 4 * (m + n + n * case["bias"]) + q * m * n * (1 + case["residual"]),
                "flops": 2 * m * n * k}
    d, h, top, local, total = (case[k] for k in ("n_model", "n_hidden", "top", "local", "total"))
    # the experts that m tokens choose, each `top` of `total` at random
    read = local * (1 - (1 - top / total) ** m)
    e = SIZES[case["dtype"]]
    moved = e * (m * d + total * d) + SIZES[case["out"]] * m * d + 8 * m * top
    moved += 3 * read * d * h * SIZES[case["weights"]]
    if case["weights"] == "int8":
        moved += 4 * read * (2 * h + d)
    return {"bytes": int(moved),
            "flops": int(2 * m * total * d + 6 * m * top * local / total * d * h)}


# ------------------------------------------------------- 64 bits, from the definition

def exact(case, seed):
    s = prepare(case, seed)
    wide = lambda t: t.to(torch.float64)  # noqa: E731
    if case["op"] == "quantise":
        x = wide(s["x"])
        most = x.abs().max(dim=1).values
        # 127 x is exact, and so is its quotient by `most` where that lies at a half
        q = torch.div(127 * x, most.clamp(min=5e-324)[:, None]).round()
        return {"q": q.to(torch.int8), "scale": most / 127}
    if case["op"] == "linear8":
        y = torch.einsum("mk,nk->mn", wide(s["x"]), wide(s["w"]))
        y = torch.einsum("mn,m,n->mn", y, wide(s["x_scale"]), wide(s["w_scale"]))
        if case["bias"]:
            y += wide(s["bias"])
        if case["residual"]:
            y += wide(s["residual"])
        return {"y": y}
    value = {
        "relu": lambda v: v.clamp(min=0),
        "gelu": lambda v: v * torch.special.ndtr(v),
        # (1 + tanh(a)) / 2 is the logistic function of 2 a
        "gelu_tanh": lambda v: v * torch.sigmoid(math.sqrt(8 / math.pi) * (v + 0.044715 * v ** 3)),
        "silu": lambda v: v * torch.sigmoid(v),
    }[case["act"]]
    x = wide(s["x"])
    logits = torch.einsum("md,ed->me", x, wide(s["router"]))
    chosen = logits.argsort(dim=1, descending=True, stable=True)[:, :case["top"]]
    if case["normalise"]:
        share = torch.softmax(logits.gather(1, chosen), dim=1)
    else:
        share = torch.softmax(logits, dim=1).gather(1, chosen)
    weights = {}
    for name in ("gate", "up", "down"):
        scale = s[name + "_scale"]
        weights[name] = lambda e, name=name, scale=scale: (
            wide(s[name][e]) if scale is None else wide(s[name][e]) * wide(scale[e])[:, None])
    y = torch.zeros_like(x)
    for e in range(case["local"]):
        token, place = (chosen == case["first"] + e).nonzero(as_tuple=True)
        if len(token):
            h = value(x[token] @ weights["gate"](e).T) * (x[token] @ weights["up"](e).T)
            y.index_add_(0, token, (h @ weights["down"](e).T) * share[token, place][:, None])
    return {"y": y, "chosen": chosen.to(torch.int32), "share": share}
