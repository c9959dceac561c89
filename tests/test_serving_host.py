"""Quantise, Linear8 and Experts without a GPU: what plans and calls refuse
before they touch the device, the binding's numbers, and the tests' own
definition of the layer against another way to compute it."""
import ctypes
import os
import re

import pytest
import torch

import test_gpu_experts as E
import test_gpu_linear8 as L8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F16, F32, I8 = 4, 5, 1, 6


@pytest.fixture(scope="module")
def pkg():
    from paper_2109_12626_gb300 import build as B
    B.build()
    import paper_2109_12626_gb300 as pkg
    pkg.lib()
    return pkg


def refused(pkg, who):
    L = pkg.lib()
    assert L.dpdr_last_error() == pkg.DPDR_ERR_INVALID
    assert who.encode() in L.dpdr_last_error_message()


@pytest.mark.parametrize("args", [(-1, 8, 8, BF16), (8, 0, 8, BF16), (8, 1 << 17, 8, BF16), (8, 8, 0, BF16),
                                  (8, 8, 1 << 31, BF16), (1 << 31, 8, 8, BF16), (8, 8, 8, I8), (8, 8, 8, 0)])
def test_integer_plans_refused(pkg, args):
    assert not pkg.lib().dpdr_integer_plan(*args)
    refused(pkg, "dpdr_integer_plan")


GOOD = dict(rows=4, d=8, h=8, experts=4, top=2, first=0, local=4, operands=BF16, weights=BF16, result=BF16, act=4, norm=1)


@pytest.mark.parametrize("bad", [
    dict(rows=0), dict(rows=65), dict(d=0), dict(h=0), dict(d=(1 << 20) + 1), dict(h=(1 << 20) + 1), dict(experts=0),
    dict(experts=513, top=1, local=1), dict(top=0), dict(top=5), dict(experts=64, top=17), dict(first=-1), dict(local=0),
    dict(first=1), dict(first=4, local=1), dict(first=2147483647, local=2), dict(operands=F32, weights=F32, result=F32),
    dict(operands=I8, weights=I8), dict(weights=F16), dict(weights=F32), dict(result=F16), dict(result=I8), dict(act=6),
    dict(act=-1)])
def test_experts_plans_refused(pkg, bad):
    assert not pkg.lib().dpdr_experts_plan(*dict(GOOD, **bad).values())
    refused(pkg, "dpdr_experts_plan")


def test_calls_without_a_plan(pkg):
    L = pkg.lib()
    for who, more in (("dpdr_integer_linear", 8), ("dpdr_experts", 12)):
        assert getattr(L, who)(None, 1, *[None] * more) == pkg.DPDR_ERR_INVALID
        refused(pkg, who)
    assert L.dpdr_integer_sync(None, None) == L.dpdr_experts_sync(None, None) == pkg.DPDR_ERR_INVALID
    L.dpdr_integer_destroy(None)
    L.dpdr_experts_destroy(None)


def matrix(at, rs, cs):
    return (ctypes.c_int64 * 3)(at, rs, cs)


@pytest.mark.parametrize("what", ["type", "n", "rows", "x", "q", "scale", "x at an odd address", "negative stride",
                                  "q turned", "q rows overlap", "overlap", "scale inside q", "too far"])
def test_quantise_refused(pkg, what):
    x, q, scale = matrix(1 << 20, 64, 1), matrix(1 << 30, 64, 1), 1 << 31
    rows, n, dtype = 8, 64, BF16
    if what == "type":
        dtype = I8
    elif what == "n":
        n = 0
    elif what == "rows":
        rows = -1
    elif what == "x":
        x = matrix(0, 64, 1)
    elif what == "scale":
        scale = None
    elif what == "x at an odd address":
        x = matrix((1 << 20) + 1, 64, 1)
    elif what == "negative stride":
        x = matrix(1 << 20, -64, 1)
    elif what == "q turned":
        q = matrix(1 << 30, 1, 8)
    elif what == "q rows overlap":
        q = matrix(1 << 30, 63, 1)
    elif what == "overlap":
        q = matrix((1 << 20) + 512, 64, 1)
    elif what == "scale inside q":
        scale = (1 << 30) + 16
    elif what == "too far":
        x = matrix(1 << 20, 1 << 58, 1)
    qa = None if what == "q" else ctypes.addressof(q)
    assert pkg.lib().dpdr_quantise(rows, n, dtype, ctypes.addressof(x), qa, scale, None) == pkg.DPDR_ERR_INVALID
    refused(pkg, "dpdr_quantise")


def test_the_binding_refuses_unknown_names(pkg):
    with pytest.raises(ValueError):
        pkg.Linear8(1, 8, 8, out="int8")
    for more in (dict(dtype="float32"), dict(weights="int4"), dict(out="int8"), dict(act="swish")):
        with pytest.raises(ValueError):
            pkg.Experts(1, 8, 8, 4, 2, **more)
    with pytest.raises(TypeError):
        pkg.quantise(torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int8), torch.zeros(2))
    with pytest.raises(TypeError):
        pkg.quantise(torch.zeros(2, 4), torch.zeros(2, 4), torch.zeros(2))
    with pytest.raises(ValueError):
        pkg.quantise(torch.zeros(2, 4), torch.zeros(2, 5, dtype=torch.int8), torch.zeros(2))
    with pytest.raises(ValueError):
        pkg.quantise(torch.zeros(2, 4, 1), torch.zeros(2, 4, dtype=torch.int8), torch.zeros(2))


def test_numbers_follow_the_header(pkg):
    from paper_2109_12626_gb300 import _native as N
    text = open(os.path.join(ROOT, "include", "dpdr.h")).read()
    assert int(re.search(r"DPDR_INT8 = (\d+)", text).group(1)) == N.DPDR_INT8
    with pytest.raises(pkg.DpdrError):
        pkg.Plan(4, 8, N.DPDR_INT8)


def layer(normalise, weights=None):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 12, generator=g).bfloat16()
    router = torch.randn(6, 12, generator=g).bfloat16()
    w = [torch.randn(6, 7, 12, generator=g).bfloat16(), torch.randn(6, 7, 12, generator=g).bfloat16(),
         torch.randn(6, 12, 7, generator=g).bfloat16()]
    return x, router, w


@pytest.mark.parametrize("normalise", [True, False])
def test_the_definition_token_by_token(normalise):
    x, router, w = layer(normalise)
    y, order, share, bound, _ = E.layer64(x, router, w, [None] * 3, 2, 0, "silu", normalise)
    for t in range(5):
        p = torch.softmax(router.double() @ x[t].double(), 0)
        s, e = p.topk(2)
        if normalise:
            s = s / s.sum()
        want = sum(s[i] * (w[2][e[i]].double() @ (torch.nn.functional.silu(w[0][e[i]].double() @ x[t].double()) *
                                                  (w[1][e[i]].double() @ x[t].double()))) for i in range(2))
        assert torch.equal(e, order[t]) and torch.allclose(s, share[t]) and torch.allclose(want, y[t])
    assert bool((bound < 1e-2 * y.abs().max()).all())


def test_a_planted_mistake_is_seen():
    x, router, w = layer(True)
    y, order, _, bound, _ = E.layer64(x, router, w, [None] * 3, 2, 0, "silu", True)
    wrong = E.layer64(x, router, [w[1], w[0], w[2]], [None] * 3, 2, 0, "silu", True)[0]
    with pytest.raises(AssertionError):
        E.U.close("y", wrong, y, bound, "float32")
    with pytest.raises(AssertionError):   # experts with lower scores are no other right choice
        E.layer64(x, router, w, [None] * 3, 2, 0, "silu", True, (order + 1) % 6)


def test_rounding_definition_at_halves():
    """Halves go to the even number: 254 x is an odd multiple of the largest size."""
    x = torch.tensor([[254.0, 1.0, 3.0, 5.0, -1.0, -3.0, 2.0]])
    q, s = L8.round64(x)
    assert q.tolist() == [[127, 0, 2, 2, 0, -2, 1]] and s.tolist() == [2.0]
