"""The bias gradient is the sum of dz before its rounding to 16 bits, with
kept projections and without."""
import pytest
import torch

import paper_2109_12626_gb300 as dpdr
import proj_util as U
from proj_tiles import tile_size

pytestmark = pytest.mark.gpu


def gen(*key):
    return torch.Generator().manual_seed(hash(key) % (1 << 31))


def sizes():
    rows, n = tile_size(152)
    return [(1, 64, 64), (2, 7, 5), (20, 136, 264), (65, 264, 71), (130, 1000, 250), (130, 2500, 129), (257, 72, 1000),
            (rows, 136, n), (rows, 72, n + 1), (20000, 40, 136), (20001, 24, 77), (70000, 8, 24)]


# The longest chain of additions behind an element: 32 rows, 64 and 8 of their
# sums, and where there are more than 512 of those as many again
CHAIN = 200 * 2.0 ** -24


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu", "sigmoid"])
@pytest.mark.parametrize("rows,k,n", sizes())
def test_as_exact_without_kept_projections(rows, k, n, act):
    """The projections that the backward call computes again are the forward
    call's bits (but of one row, whose forward product is a kernel of its own),
    so both ways add up the same float32 dz, in another order."""
    for dtype in ("bfloat16", "float16"):
        g = gen(rows, k, n, dtype == "float16")
        x, w = U.matrix(g, rows, k, dtype), U.matrix(g, n, k, dtype, scale=k ** -0.5)
        b, dy = U.matrix(g, 1, n, dtype).reshape(-1), U.matrix(g, rows, n, dtype)
        pre, y = torch.empty(rows, n, device="cuda"), torch.empty(rows, n, dtype=U.TYPES[dtype], device="cuda")
        kept, again, half = (torch.full((n,), 9.0, device="cuda") for _ in range(3))
        half = half.to(U.TYPES[dtype])
        with dpdr.Linear(rows + 2, k, n, dtype, grad="float32", act=act) as plan, dpdr.Linear(rows, k, n, dtype, act=act) as p16:
            plan.forward(x, w, y, bias=b, pre=pre)
            plan.backward(x, w, dy, dbias=kept, bias=b, pre=pre)
            plan.backward(x, w, dy, dbias=again, bias=b)
            p16.backward(x, w, dy, dbias=half, bias=b)
            plan.sync()
            p16.sync()
        sizes = (dy.double() * U.slope64(act, pre.double())).abs().sum(0)
        off = (kept.double() - again.double()).abs()
        if rows == 1:
            z, of_z = U.linear64(x, w, b, act)
            off -= 2 * (dy.double().abs() * U.slope_bound(act, z, of_z)[1]).sum(0)
        assert bool((off <= 2 * CHAIN * sizes + 1e-30).all()), (dtype, (off / sizes).max().item())
        U.close("16 bits", half, again.double(), 1e-30 * sizes, dtype)


@pytest.mark.parametrize("scale", [1e6, 1e-9])
@pytest.mark.parametrize("rows,k,n", [(20, 136, 264), (1300, 72, 1501), (20000, 40, 136)])
def test_beyond_the_operands_range(rows, k, n, scale):
    """Float32 dy so large or small that dz as float16 is infinite or 0."""
    g = gen(rows, n)
    x, w = U.matrix(g, rows, k, "float16"), U.matrix(g, n, k, "float16", scale=k ** -0.5)
    dy = (torch.rand(rows, n, generator=g) + 0.5).cuda() * scale
    db = torch.empty(n, device="cuda")
    with dpdr.Linear(rows, k, n, "float16", out="float32", grad="float32", act="sigmoid") as plan:
        plan.backward(x, w, dy, dbias=db)
        plan.sync()
    z, off = U.linear64(x, w, None, "sigmoid")
    s, e = U.slope_bound("sigmoid", z, off)
    want = (dy.double() * s).sum(0)
    assert bool(((db.double() - want).abs() <= (dy.double() * e).sum(0) + CHAIN * want).all())


def test_the_same_bits():
    for rows, k, n in ((130, 1000, 250), (20001, 24, 77), tile_size(152) + (72,)):
        g = gen(rows)
        x, w, dy = U.matrix(g, rows, k, "bfloat16"), U.matrix(g, n, k, "bfloat16"), U.matrix(g, rows, n, "bfloat16")
        a, b = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        with dpdr.Linear(rows, k, n, grad="float32", act="silu") as plan:
            plan.backward(x, w, dy, dbias=a)
            plan.backward(x, w, dy, dbias=b)
            plan.sync()
        assert torch.equal(a, b)
