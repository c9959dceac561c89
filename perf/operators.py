"""Performance cases of the projections around a reduction-to-all: a matrix
product with bias, activation and residual (``linear``) and a gated pair of
projections (``gated``), forward alone or with their gradients.

A case names the operator (``op``), whether a pass is the forward call or a
training step's forward and backward calls (``train``), the sizes, the operand
type, the activation, the result's and the gradients' types, and how the data
lies: ``turned`` weights are held as [in, out] and passed as a transposed
view, ``slack`` rows of x are that many elements apart more than they are
long (a slice of a wider array).  ``keep``: the forward pass keeps its
projections before the activation for the backward pass, which otherwise
computes them again.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}


def _case(name, op, rows, n_in, n_out, dtype="bfloat16", act="none", train=False, out=None,
          grad=None, bias=False, residual=False, keep=False, turned=False, slack=0):
    return {"name": name, "op": op, "train": train, "rows": rows, "n_in": n_in, "n_out": n_out,
            "dtype": dtype, "act": act, "out": out or dtype, "grad": grad or dtype, "bias": bias,
            "residual": residual, "keep": keep, "turned": turned, "slack": slack}


def listed():
    return [
        # one token of one sequence being answered, the residual stream added
        _case("linear_token", "linear", 1, 4096, 4096, residual=True),
        # a small batch of sequences being answered: one rank's share of a
        # row-parallel projection, as the float32 partial that ranks add up
        _case("linear_partial_24_rows", "linear", 24, 1024, 8192, "float16", out="float32"),
        # a short prompt through odd sizes
        _case("linear_ragged", "linear", 333, 2500, 1000, act="gelu", bias=True, residual=True),
        # a long prompt or a large batch
        _case("linear_prompt", "linear", 8192, 8192, 4096, bias=True, residual=True),
        # a training step of a projection with its activation
        _case("linear_training", "linear", 4096, 4096, 4096, act="gelu_tanh", train=True,
              bias=True, keep=True),
        # a training step at odd sizes whose gradients are added up over
        # data-parallel ranks in float32
        _case("linear_training_odd", "linear", 1000, 4100, 2500, "float16", train=True, bias=True,
              grad="float32"),
        # the same pair of projections for one token
        _case("gated_token", "gated", 1, 4096, 8192, act="silu"),
        # a batch of sequences being answered
        _case("gated_48_rows", "gated", 48, 5120, 2048, "float16", act="gelu_tanh"),
        # odd sizes, weights held the other way round
        _case("gated_ragged", "gated", 777, 1000, 4099, act="silu", turned=True),
        # a long prompt or a large batch
        _case("gated_prompt", "gated", 8192, 4096, 8192, act="silu"),
        # a training step
        _case("gated_training", "gated", 4096, 4096, 8192, act="silu", train=True, keep=True),
        # a small training step that keeps nothing between the passes
        _case("gated_training_small", "gated", 130, 1000, 2500, "float16", act="gelu", train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "gated"])
    train = rng.random() < 0.4
    rows = _log(rng, 1, 8192)
    n_in, n_out = _log(rng, 64, 8192), _log(rng, 64, 8192)
    how = rng.random()
    if how < 0.6:  # sizes as models have them: multiples of 64; else as drawn
        n_in, n_out = max(64, n_in // 64 * 64), max(64, n_out // 64 * 64)
        if how < 0.3:
            rows = max(1, rows // 8 * 8)
    act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"] if op == "linear"
                     else ["silu", "silu", "gelu", "gelu_tanh", "relu"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16"])
    out = "float32" if op == "linear" and not train and rng.random() < 0.4 else dtype
    grad = "float32" if op == "linear" and act == "none" and rng.random() < 0.5 else dtype
    c = _case("", op, rows, n_in, n_out, dtype, act, train, out, grad,
              bias=op == "linear" and rng.random() < 0.6,
              residual=op == "linear" and not train and rng.random() < 0.5,
              keep=train and act != "none" and rng.random() < 0.6, turned=rng.random() < 0.2,
              slack=rng.choice([0, 0, 0, 8, 11]))
    del c["name"]
    while work(c)["flops"] > 1.1e12:
        c["rows"] //= 2
    return c


def _weight(case, g, rows):
    """[rows, n_in], of rows as long as one for variance 1/n_in."""
    shape = (case["n_in"], rows) if case["turned"] else (rows, case["n_in"])
    w = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda")
    w.normal_(0.0, case["n_in"] ** -0.5, generator=g)
    return w.t() if case["turned"] else w


def _normal(g, shape, dtype, scale=1.0):
    return torch.empty(shape, dtype=DTYPES[dtype], device="cuda").normal_(0.0, scale, generator=g)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    m, k, n = case["rows"], case["n_in"], case["n_out"]
    linear, dt, out, grad = case["op"] == "linear", case["dtype"], case["out"], case["grad"]
    new = lambda shape, d: torch.empty(shape, dtype=DTYPES[d], device="cuda")  # noqa: E731
    s = {"case": case}
    s["x"] = _normal(g, (m, k + case["slack"]), dt)[:, :k]
    s["w"] = [_weight(case, g, n) for _ in range(1 if linear else 2)]
    s["bias"] = _normal(g, (n,), dt, 0.1) if case["bias"] else None
    s["residual"] = _normal(g, (m, n), out) if case["residual"] else None
    s["dy"] = _normal(g, (m, n), out) if case["train"] else None
    # buffers that the program holds for the results
    s["y"] = new((m, n), out)
    if case["train"]:
        s["pre"] = new((m, n if linear else 2 * n), "float32") if case["keep"] else None
        s["dx"], s["dw"] = new((m, k), grad), [new((n, k), grad) for _ in s["w"]]
        s["dbias"] = new((n,), grad) if case["bias"] else None
    if own:
        import paper_2109_12626_gb300 as pkg
        make = pkg.Linear if linear else pkg.Gated
        s["plan"] = make(m, k, n, dt, out=out, grad=grad, act=case["act"])
    return s


# ------------------------------------------------------- the plain form

_ROOT_2_PI, _CUBIC = math.sqrt(2.0 / math.pi), 0.044715


def _act(name, z):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_ROOT_2_PI * (z + _CUBIC * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) \
            + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(_ROOT_2_PI * (z + _CUBIC * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _ROOT_2_PI * (1 + 3 * _CUBIC * z * z)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain(s):
    case, act = s["case"], s["case"]["act"]
    out, grad = DTYPES[case["out"]], DTYPES[case["grad"]]
    x, w = s["x"].float(), [v.float() for v in s["w"]]
    z = [x @ v.t() for v in w]
    if s["bias"] is not None:
        z[0] = z[0] + s["bias"].float()
    y = _act(act, z[0])
    if case["op"] == "gated":
        y = y * z[1]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not case["train"]:
        return {"y": y.to(out)}
    dy = s["dy"].float()
    if case["op"] == "gated":
        dz = [dy * z[1] * _slope(act, z[0]), dy * _act(act, z[0])]
    else:
        dz = [dy * _slope(act, z[0]) if act != "none" else dy]
    dx = dz[0] @ w[0] if len(w) == 1 else dz[0] @ w[0] + dz[1] @ w[1]
    return {"y": y.to(out), "dx": dx.to(grad), "dw": [(d.t() @ x).to(grad) for d in dz],
            "dbias": dz[0].sum(0).to(grad) if s["bias"] is not None else None}


# ----------------------------------------------------- the framework's calls

def _own(s):
    case, plan, train = s["case"], s["plan"], s["case"]["train"]
    pre = s["pre"] if train else None
    if case["op"] == "linear":
        plan.forward(s["x"], s["w"][0], s["y"], bias=s["bias"], residual=s["residual"], pre=pre)
        if not train:
            return {"y": s["y"]}
        plan.backward(s["x"], s["w"][0], s["dy"], dx=s["dx"], dw=s["dw"][0], dbias=s["dbias"],
                      bias=s["bias"], pre=pre)
    else:
        plan.forward(s["x"], s["w"][0], s["w"][1], s["y"], pre=pre)
        if not train:
            return {"y": s["y"]}
        plan.backward(s["x"], s["w"][0], s["w"][1], s["dy"], dx=s["dx"], dw_gate=s["dw"][0],
                      dw_up=s["dw"][1], pre=pre)
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------- its work

def work(case):
    m, k, n = case["rows"], case["n_in"], case["n_out"]
    size = {"bfloat16": 2, "float16": 2, "float32": 4}
    e, s, q = size[case["dtype"]], size[case["out"]], size[case["grad"]]
    pair = 1 if case["op"] == "linear" else 2
    moved = e * (m * k + pair * n * k + n * case["bias"]) + s * m * n * (1 + case["residual"])
    flops = 2 * pair * m * n * k
    if case["train"]:
        moved += s * m * n + q * (m * k + pair * n * k + n * case["bias"])
        flops *= 3
    return {"bytes": moved, "flops": flops}


# ------------------------------------------------------- 64 bits, from the definition

def exact(case, seed):
    s = prepare(case, seed)
    wide = lambda t: t.to(torch.float64)  # noqa: E731
    phi = lambda v: torch.special.ndtr(v)  # noqa: E731, the normal distribution
    c = 2 * _ROOT_2_PI
    value, slope = {
        "none": (lambda v: v, torch.ones_like),
        "relu": (lambda v: v.clamp(min=0), lambda v: torch.heaviside(v, torch.zeros_like(v))),
        "gelu": (lambda v: v * phi(v), lambda v: phi(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)),
        # (1 + tanh(a)) / 2 is the logistic function of 2 a
        "gelu_tanh": (lambda v: v * torch.sigmoid(c * (v + _CUBIC * v ** 3)),
                      lambda v: torch.sigmoid(c * (v + _CUBIC * v ** 3)) * (
                          1 + v * c * (1 + 3 * _CUBIC * v ** 2) * torch.sigmoid(-c * (v + _CUBIC * v ** 3)))),
        "silu": (lambda v: v * torch.sigmoid(v),
                 lambda v: torch.sigmoid(v) * (1 + v * torch.sigmoid(-v))),
    }[case["act"]]
    x, first = wide(s["x"]), wide(s["w"][0])
    z = torch.einsum("mk,nk->mn", x, first)
    if case["bias"]:
        z += wide(s["bias"])
    got = {"dbias": None}
    if case["op"] == "linear":
        got["y"] = value(z) + (wide(s["residual"]) if case["residual"] else 0.0)
        if case["train"]:
            dz = wide(s["dy"]) * slope(z)
            got["dx"] = torch.einsum("mn,nk->mk", dz, first)
            got["dw"] = [torch.einsum("mn,mk->nk", dz, x)]
            got["dbias"] = dz.sum(dim=0) if case["bias"] else None
    else:
        second = wide(s["w"][1])
        u = torch.einsum("mk,nk->mn", x, second)
        got["y"] = value(z) * u
        if case["train"]:
            dh = wide(s["dy"])
            dg, du = dh * u * slope(z), dh * value(z)
            got["dx"] = torch.einsum("mn,nk->mk", dg, first) + torch.einsum("mn,nk->mk", du, second)
            got["dw"] = [torch.einsum("mn,mk->nk", d, x) for d in (dg, du)]
    if not case["train"]:
        del got["dbias"]
    return got
