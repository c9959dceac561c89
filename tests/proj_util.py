"""The projections' definition in 64 bits with bounds on what a right kernel
may be off by, and inputs laid out in several ways."""
from __future__ import annotations

import math

import torch

TYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}
# unit roundoff of a result; 0 for float32, whose rounding is far below the sum's
ROUND = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -23}
# the least positive value times one half: what rounding to float16 may be off
# by below its normal range (the other types' ranges are not left here)
TINY = {"bfloat16": 1e-38, "float16": 2.0 ** -25, "float32": 1e-38}
LIPSCHITZ = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "gelu_tanh": 1.13, "silu": 1.1, "sigmoid": 0.25}
CURVE = {"none": 0.0, "relu": 0.0, "gelu": 0.8, "gelu_tanh": 0.85, "silu": 0.5, "sigmoid": 0.1}


def act64(name, z):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "sigmoid":
        return torch.sigmoid(z)
    return z


def slope64(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    z = z.detach().clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(act64(name, z).sum(), z)[0]


def summed(k):
    """Relative error of a float32 sum of k products, of the sum of their
    sizes, in any order: one unit roundoff an addition, of 2^-23 where sums
    are cut off instead of rounded, twice that for products that are aligned
    before they are added."""
    return (k + 8) * 2.0 ** -22


# relative error of an activation and of its slope as float32 code, which
# takes a handful of operations of 2^-22 each and one exp or erfc
EVAL = 2.0 ** -18


def linear64(x, w, bias, act):
    """z, and the bound of a float32 z."""
    x, w = x.double(), w.double()
    z = x @ w.t()
    off = summed(x.shape[1]) * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.double()
        off = off + 2.0 ** -23 * z.abs()
    return z, off


def close(name, got, want, bound, out):
    """got within bound (and its own rounding) of want, element by element."""
    assert got.shape == want.shape, name
    far = (got.double() - want).abs() - (bound + ROUND[out] * want.abs() * 1.01 + TINY[out])
    bad = ~(far <= 0)
    assert not bool(bad.any()), "%s: %d of %d too far, worst %.3g at a value of %.3g" % (
        name, int(bad.sum()), far.numel(), float(far.max()), float(want.reshape(-1)[far.reshape(-1).argmax()]))


def close_in_norm(name, got, want, rel):
    d, n = (got.double() - want).norm().item(), want.norm().item()
    assert d <= rel * n + 1e-30, "%s: off by %.3g of its norm, %.3g allowed" % (name, d / max(n, 1e-300), rel)


def check_linear(got_y, x, w, bias, residual, act, out, pre=None):
    z, off = linear64(x, w, bias, act)
    if pre is not None:
        close("pre", pre, z, off, "float32")
    y = act64(act, z)
    off = LIPSCHITZ[act] * off + EVAL * y.abs() + 1e-30
    if residual is not None:
        y = y + residual.double()
    close("y", got_y, y, off + 2.0 ** -22 * y.abs(), out)
    if x.shape[0] * w.shape[0] >= 1000:   # random roundings: no more than one unit in the norm
        close_in_norm("y", got_y, y, ROUND[out] + 2.0 ** -17)


def check_gated(got_h, x, wg, wu, act, out, pre=None):
    g, eg = linear64(x, wg, None, act)
    u, eu = linear64(x, wu, None, act)
    if pre is not None:
        close("pre", pre, torch.cat([g, u], 1), torch.cat([eg, eu], 1), "float32")
    a = act64(act, g)
    ea = LIPSCHITZ[act] * eg + EVAL * a.abs() + 1e-30
    close("h", got_h, a * u, ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -22 * (a * u).abs(), out)
    if g.numel() >= 1000:
        close_in_norm("h", got_h, a * u, ROUND[out] + 2.0 ** -17)


def check_products(dz, edz, ws, x, dtype, grad, got_dx, got_dw, got_db):
    """dx, dw and dbias from each dz with its bound; dz is rounded to dtype."""
    edz = [e + ROUND[dtype] * (d.abs() + e) * 1.01 + TINY[dtype] for d, e in zip(dz, edz)]
    big = [d.abs() + e for d, e in zip(dz, edz)]
    norm = ROUND[grad] + 2 * ROUND[dtype] + 2.0 ** -17   # dz rounded and sums of such
    if got_dx is not None:
        k = summed(sum(w.shape[0] for w in ws))
        want = sum(d @ w.double() for d, w in zip(dz, ws))
        close("dx", got_dx, want, sum((e + k * b) @ w.double().abs() for e, b, w in zip(edz, big, ws)), grad)
        if want.numel() >= 1000:
            close_in_norm("dx", got_dx, want, norm)
    for i, got in enumerate(got_dw or []):
        want = dz[i].t() @ x.double()
        close("dw", got, want, (edz[i] + summed(x.shape[0]) * big[i]).t() @ x.double().abs(), grad)
        if want.numel() >= 1000:
            close_in_norm("dw", got, want, norm)
    if got_db is not None:
        close("dbias", got_db, dz[0].sum(0), (edz[0] + summed(x.shape[0]) * big[0]).sum(0), grad)


def slope_bound(act, z, off):
    """act'(z) for a z that is off by `off`, and what it may be off by."""
    s = slope64(act, z)
    e = CURVE[act] * off + EVAL * (1 + s.abs())
    if act == "relu":   # a z next to 0 may fall on either side
        e = e + (z.abs() <= off).to(z.dtype)
    return s, e


def check_linear_gradients(x, w, bias, dy, act, dtype, grad, dx=None, dw=None, dbias=None):
    z, off = linear64(x, w, bias, act)
    s, e = slope_bound(act, z, off)
    dy = dy.double()
    check_products([dy * s], [dy.abs() * e], [w], x, dtype, grad, dx, [dw] if dw is not None else None, dbias)


def check_gated_gradients(x, wg, wu, dh, act, dtype, grad, dx=None, dw=None):
    g, eg = linear64(x, wg, None, act)
    u, eu = linear64(x, wu, None, act)
    s, es = slope_bound(act, g, eg)
    a = act64(act, g)
    ea = LIPSCHITZ[act] * eg + EVAL * a.abs() + 1e-30
    dh = dh.double()
    check_products([dh * u * s, dh * a],
                   [dh.abs() * (es * (u.abs() + eu) + s.abs() * eu + 2.0 ** -21 * (u * s).abs()),
                    dh.abs() * (ea + 2.0 ** -22 * a.abs())],
                   [wg, wu], x, dtype, grad, dx, dw, None)


# ------------------------------------------------------------------ inputs

def matrix(g, rows, cols, dtype, how="plain", scale=1.0):
    """A seeded normal matrix: "plain" rows, "turned" (a transposed view),
    "slack" (a slice of a wider array, 8 more a row), "odd" (a slice 3 wider
    that starts one element in), or "apart" (neither stride is 1)."""
    t = TYPES[dtype]
    rnd = lambda *s: (torch.randn(*s, generator=g) * scale).to(t)  # noqa: E731
    if how == "turned":
        return rnd(cols, rows).cuda().t()
    if how == "slack":
        return rnd(rows, cols + 8).cuda()[:, :cols]
    if how == "odd":
        return rnd(rows, cols + 3).cuda()[:, 1:cols + 1]
    if how == "apart":
        return rnd(rows, 2 * cols).cuda()[:, ::2]
    return rnd(rows, cols).cuda()


class Guarded:
    """A result of rows x cols inside a wider array of a known value, which
    must still be there around it afterwards."""

    def __init__(self, rows, cols, dtype, left=8, right=8, above=1):
        self.value = -77.0
        self.base = torch.full((rows + 2 * above, left + cols + right), self.value, dtype=TYPES[dtype], device="cuda")
        self.t = self.base[above:above + rows, left:left + cols]

    def check(self):
        inside = self.t.clone()
        self.t.fill_(self.value)
        assert bool((self.base == self.value).all()), "written outside of the result"
        self.t.copy_(inside)
        return self.t
