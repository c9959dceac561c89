"""The projections without a GPU: what plans and calls refuse before they
touch the device, the binding's numbers against the header's, and the tests'
own definition in 64 bits against automatic differentiation."""
import os
import re

import pytest
import torch

import proj_util as U

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pkg():
    from paper_2109_12626_gb300 import build as B
    B.build()
    import paper_2109_12626_gb300 as pkg
    pkg.lib()
    return pkg


BF16, F16, F32 = 4, 5, 1


@pytest.mark.parametrize("make", ["dpdr_linear_plan", "dpdr_gated_plan"])
@pytest.mark.parametrize("args", [
    (-1, 8, 8, BF16, BF16, BF16, 0), (8, 0, 8, BF16, BF16, BF16, 0), (8, 8, 0, BF16, BF16, BF16, 0),
    (1 << 31, 8, 8, BF16, BF16, BF16, 0), (8, 1 << 31, 8, BF16, BF16, BF16, 0), (8, 8, -5, BF16, BF16, BF16, 0),
    (8, 8, 8, F32, F32, F32, 0), (8, 8, 8, 0, 0, 0, 0), (8, 8, 8, BF16, F16, BF16, 0), (8, 8, 8, BF16, BF16, F16, 0),
    (8, 8, 8, F16, F16, 2, 0), (8, 8, 8, BF16, BF16, BF16, 6), (8, 8, 8, BF16, BF16, BF16, -1)])
def test_plans_refused(pkg, make, args):
    L = pkg.lib()
    assert not getattr(L, make)(*args)
    assert L.dpdr_last_error() == pkg.DPDR_ERR_INVALID
    assert make.encode() in L.dpdr_last_error_message()


def test_calls_without_a_plan(pkg):
    L = pkg.lib()
    for rc in (L.dpdr_linear(None, 1, *[None] * 7), L.dpdr_gated(None, 1, *[None] * 6),
               L.dpdr_linear_backward(None, 1, *[None] * 9), L.dpdr_gated_backward(None, 1, *[None] * 9),
               L.dpdr_proj_sync(None, None)):
        assert rc == pkg.DPDR_ERR_INVALID
    L.dpdr_proj_destroy(None)


def test_reductions_do_not_take_the_operand_types(pkg):
    for t in (BF16, F16):
        with pytest.raises(pkg.DpdrError):
            pkg.Plan(4, 8, t)


def test_numbers_follow_the_header(pkg):
    from paper_2109_12626_gb300 import projections as P
    text = open(os.path.join(ROOT, "include", "dpdr.h")).read()
    values = {k: int(v) for k, v in re.findall(r"\b(DPDR_[A-Z0-9_]+) = (\d+)", text)}
    for name, v in P.ACTIVATIONS.items():
        assert values["DPDR_ACT_" + name.upper()] == v
    for name, v in P.RESULTS.items():
        assert values["DPDR_" + name.upper()] == v


@pytest.mark.parametrize("act", list(U.LIPSCHITZ))
def test_bounds_of_the_activations(act):
    """The Lipschitz constants and curvatures that the tests' bounds use hold
    on a fine grid, and the slopes are those of automatic differentiation."""
    z = torch.linspace(-12, 12, 200001, dtype=torch.float64)
    s = U.slope64(act, z)
    assert s.abs().max() <= U.LIPSCHITZ[act] * 1.001
    if act != "relu":   # its slope jumps at 0, which the bounds treat apart
        assert ((s[1:] - s[:-1]).abs() / (z[1] - z[0])).max() <= U.CURVE[act] + 1e-3
    v = U.act64(act, z)
    d = (v[2:] - v[:-2]) / (z[2] - z[0])
    off = z[1:-1].abs() > 1e-3 if act == "relu" else slice(None)
    assert (d - s[1:-1])[off].abs().max() < 1e-7


def test_the_definition_against_automatic_differentiation():
    g = torch.Generator().manual_seed(3)
    x, wg, wu = (torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_(True) for s in ((5, 7), (6, 7), (6, 7)))
    dh = torch.randn(5, 6, generator=g, dtype=torch.float64)
    dx, dg, du = torch.autograd.grad((dh * U.act64("silu", x @ wg.t()) * (x @ wu.t())).sum(), (x, wg, wu))
    U.check_gated_gradients(x.detach(), wg.detach(), wu.detach(), dh, "silu", "float16", "float32", dx, [dg, du])
    b = torch.randn(6, generator=g, dtype=torch.float64).requires_grad_(True)
    dx, dw, db = torch.autograd.grad((dh * U.act64("gelu", x @ wg.t() + b)).sum(), (x, wg, b))
    U.check_linear_gradients(x.detach(), wg.detach(), b.detach(), dh, "gelu", "float16", "float32", dx, dw, db)
    with pytest.raises(AssertionError):   # a mistake in a gradient is seen
        U.check_linear_gradients(x.detach(), wg.detach(), b.detach(), dh, "gelu", "float16", "float32", dx, dw.flip(0), db)


def test_kernels_wait_by_warps():
    """What follows a wait in the kernels (loads from tensor memory, barriers
    of the CTA) is for whole warps, so they never take a lane's own answer."""
    csrc = os.path.join(ROOT, "paper_2109_12626_gb300", "csrc")
    for name in ("proj_tile.cuh", "proj_rows.cuh"):
        text = open(os.path.join(csrc, name)).read()
        assert "bar_wait_warp(" in text and not re.search(r"\bbar_wait\(", text), name


def test_a_cta_settles_before_it_leaves():
    """Loads and products may be under way when a wait has run out, asked for
    by either loading warp of either CTA of a pair: a CTA with a failed wait
    settles after the last of its warps has ended and before it frees tensor
    memory or leaves."""
    csrc = os.path.join(ROOT, "paper_2109_12626_gb300", "csrc")
    for name, pattern in (("proj_tile.cuh", r"__syncthreads\(\);\s+if \(stop\) settle\(\);\s+cluster_sync\(\);"),
                          ("proj_rows.cuh", r"ok = __syncthreads_and\(ok && !stop\);[^\n]*\s+if \(!ok\) settle\(\);")):
        text = open(os.path.join(csrc, name)).read()
        at = re.search(pattern, text)
        assert at and text.index("tmem_free<") > at.end(), name
