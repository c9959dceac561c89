"""The projections (Linear, Gated) against their definition in 64 bits: sizes
from one row and column on, odd ones, every type, activation and way the
data may lie; gradients against the formulas and against differences."""
import ctypes

import pytest
import torch

import paper_2109_12626_gb300 as dpdr
import proj_util as U

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid"]


def gen(*key):
    return torch.Generator().manual_seed(hash(key) % (1 << 31))


def linear_case(rows, k, n, dtype="bfloat16", out=None, act="none", bias=True, residual=True, lay=("plain", "plain"),
                pre=False, guard=(8, 8)):
    g = gen(rows, k, n)
    out = out or dtype
    x = U.matrix(g, rows, k, dtype, lay[0])
    w = U.matrix(g, n, k, dtype, lay[1], k ** -0.5)
    b = U.matrix(g, 1, n, dtype).reshape(-1) if bias else None
    r = U.matrix(g, rows, n, out) if residual else None
    y = U.Guarded(rows, n, out, *guard)
    p = U.Guarded(rows, n, "float32") if pre else None
    with dpdr.Linear(rows + 3, k, n, dtype, out=out, act=act) as plan:
        plan.forward(x, w, y.t, bias=b, residual=r, pre=p.t if pre else None)
        plan.sync()
        U.check_linear(y.check(), x, w, b, r, act, out, p.check() if pre else None)


SIZES = [(1, 64, 64), (1, 1, 1), (1, 4096, 136), (2, 7, 5), (3, 8, 129), (5, 100, 8), (8, 72, 1000), (16, 1000, 96),
         (17, 513, 259), (33, 65, 200), (64, 256, 128), (65, 264, 72), (127, 128, 385), (129, 96, 264),
         (130, 1000, 250), (200, 40, 24), (256, 64, 512), (257, 2500, 130), (300, 129, 1), (513, 72, 513),
         (1025, 192, 640), (1, 136, 70000), (70000, 24, 40)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_linear_sizes(rows, k, n, dtype):
    linear_case(rows, k, n, dtype)


@pytest.mark.parametrize("rows,k,n", [(1, 520, 264), (24, 1024, 513), (160, 200, 328), (700, 264, 520)])
@pytest.mark.parametrize("act", ACTS)
def test_linear_activations_with_kept_projection(rows, k, n, act):
    linear_case(rows, k, n, act=act, pre=True)
    linear_case(rows, k, n, act=act, out="float32", residual=False, bias=False)


@pytest.mark.parametrize("rows,k,n", [(4, 136, 264), (40, 128, 72), (333, 250, 1000), (600, 264, 136)])
@pytest.mark.parametrize("lx", ["plain", "turned", "slack", "odd", "apart"])
@pytest.mark.parametrize("lw", ["plain", "turned", "slack", "odd", "apart"])
def test_linear_layouts(rows, k, n, lx, lw):
    linear_case(rows, k, n, lay=(lx, lw))


@pytest.mark.parametrize("out", ["float16", "float32"])
@pytest.mark.parametrize("guard", [(1, 2), (2, 2), (4, 5), (3, 0)])
@pytest.mark.parametrize("rows,n", [(1, 8), (3, 130), (70, 264), (300, 520)])
def test_linear_result_places(out, guard, rows, n):
    linear_case(rows, 72, n, "float16", out=out, guard=guard)


@pytest.mark.parametrize("rows,k,n", [(1, 64, 72), (50, 64, 130), (400, 136, 264)])
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_linear_onto_its_residual(rows, k, n, out):
    g = gen(rows, n, 1)
    x, w = U.matrix(g, rows, k, "bfloat16"), U.matrix(g, n, k, "bfloat16", scale=k ** -0.5)
    y = U.Guarded(rows, n, out)
    r = U.matrix(g, rows, n, out)
    y.t.copy_(r)
    with dpdr.Linear(rows, k, n, "bfloat16", out=out, act="silu") as plan:
        plan.forward(x, w, y.t, residual=y.t)
        plan.sync()
    U.check_linear(y.check(), x, w, None, r, "silu", out)


def test_linear_residual_as_broadcast_and_turned():
    g = gen(9)
    x, w = U.matrix(g, 40, 64, "bfloat16"), U.matrix(g, 136, 64, "bfloat16", scale=0.125)
    y = torch.empty(40, 136, dtype=torch.bfloat16, device="cuda")
    for r in (U.matrix(g, 1, 136, "bfloat16").expand(40, 136), U.matrix(g, 40, 1, "bfloat16").expand(40, 136),
              U.matrix(g, 40, 136, "bfloat16", "turned")):
        with dpdr.Linear(40, 64, 136) as plan:
            plan.forward(x, w, y, residual=r)
            plan.sync()
        U.check_linear(y, x, w, None, r, "none", "bfloat16")


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_gated_sizes(rows, k, n, dtype):
    gated_case(rows, k, n, dtype)


def gated_case(rows, k, n, dtype="bfloat16", act="silu", out=None, lay=("plain", "plain", "plain"), pre=False,
               guard=(8, 8)):
    g = gen(rows, k, n, 2)
    out = out or dtype
    x = U.matrix(g, rows, k, dtype, lay[0])
    wg, wu = (U.matrix(g, n, k, dtype, lay[i], k ** -0.5) for i in (1, 2))
    h = U.Guarded(rows, n, out, *guard)
    p = U.Guarded(rows, 2 * n, "float32") if pre else None
    with dpdr.Gated(rows, k, n, dtype, out=out, act=act) as plan:
        plan.forward(x, wg, wu, h.t, pre=p.t if pre else None)
        plan.sync()
        U.check_gated(h.check(), x, wg, wu, act, out, p.check() if pre else None)


# long sums and few tiles, where the parts of a sum are many; the last has 128 columns
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,k,n", [(2, 2500, 300), (40, 3333, 700), (64, 8192, 512), (100, 5000, 2900),
                                      (150, 4097, 600), (300, 2560, 1000), (520, 6150, 1200)])
def test_long_sums(rows, k, n, out):
    linear_case(rows, k, n, out=out, act="silu", pre=True)
    gated_case(rows, k, (n + 1) // 2, out=out, act="gelu_tanh")


@pytest.mark.parametrize("rows,k,n", [(1, 520, 264), (24, 1024, 513), (160, 200, 328), (700, 264, 520)])
@pytest.mark.parametrize("act", ACTS)
def test_gated_activations_with_kept_projections(rows, k, n, act):
    gated_case(rows, k, n, act=act, pre=True)
    gated_case(rows, k, n, act=act, out="float32", guard=(3, 2))


@pytest.mark.parametrize("rows,k,n", [(4, 136, 264), (40, 128, 72), (600, 250, 136)])
@pytest.mark.parametrize("lay", [("plain", "turned", "turned"), ("turned", "plain", "plain"), ("odd", "plain", "turned"),
                                 ("plain", "odd", "plain"), ("slack", "slack", "apart"), ("apart", "turned", "odd")])
def test_gated_layouts(rows, k, n, lay):
    gated_case(rows, k, n, lay=lay)


def test_gated_weights_as_halves_of_one_array():
    g = gen(4)
    both = U.matrix(g, 2 * 200, 136, "bfloat16", scale=0.1)
    x = U.matrix(g, 77, 136, "bfloat16")
    h = torch.empty(77, 200, dtype=torch.bfloat16, device="cuda")
    for wg, wu in ((both[:200], both[200:]), (both[0::2], both[1::2])):
        with dpdr.Gated(77, 136, 200) as plan:
            plan.forward(x, wg, wu, h)
            plan.sync()
        U.check_gated(h, x, wg, wu, "silu", "bfloat16")


# ---------------------------------------------------------------- gradients

GRAD_SIZES = [(1, 64, 64), (1, 1, 1), (2, 7, 5), (3, 136, 70), (16, 72, 264), (65, 264, 72), (130, 1000, 250),
              (256, 512, 128), (333, 100, 259), (1000, 136, 200), (2049, 24, 40), (5, 4100, 130), (6, 72, 5000)]


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("rows,k,n", GRAD_SIZES)
def test_linear_gradients(rows, k, n, act, keep):
    linear_gradient_case(rows, k, n, act=act, keep=keep)


def linear_gradient_case(rows, k, n, dtype="bfloat16", out=None, grad=None, act="none", keep=False, bias=True,
                         lay=("plain", "plain", "plain"), what=("dx", "dw", "dbias")):
    g = gen(rows, k, n, 3)
    out, grad = out or dtype, grad or dtype
    x, w = U.matrix(g, rows, k, dtype, lay[0]), U.matrix(g, n, k, dtype, lay[1], k ** -0.5)
    b = U.matrix(g, 1, n, dtype).reshape(-1) if bias else None
    dy = U.matrix(g, rows, n, out, lay[2])
    res = {"dx": U.Guarded(rows, k, grad), "dw": U.Guarded(n, k, grad), "dbias": U.Guarded(1, n, grad)}
    with dpdr.Linear(rows + 5, k, n, dtype, out=out, grad=grad, act=act) as plan:
        pre = None
        if keep:
            pre = torch.empty(rows, n, device="cuda")
            plan.forward(x, w, torch.empty(rows, n, dtype=U.TYPES[out], device="cuda"), bias=b, pre=pre)
        plan.backward(x, w, dy, bias=b, pre=pre, **{m: res[m].t.reshape(-1) if m == "dbias" else res[m].t for m in what})
        plan.sync()
    got = {m: res[m].check() for m in what}
    if "dbias" in got:
        got["dbias"] = got["dbias"].reshape(-1)
    U.check_linear_gradients(x, w, b, dy, act, dtype, grad, **got)


@pytest.mark.parametrize("act", ACTS)
def test_linear_gradients_of_activations(act):
    linear_gradient_case(150, 200, 136, "float16", act=act)
    linear_gradient_case(150, 200, 136, "bfloat16", grad="float32", act=act, keep=True)


@pytest.mark.parametrize("rows,k,n", [(1, 72, 136), (20, 136, 72), (300, 264, 136)])
@pytest.mark.parametrize("lay", [("turned", "plain", "plain"), ("plain", "turned", "plain"), ("odd", "odd", "odd"),
                                 ("plain", "plain", "turned"), ("apart", "slack", "apart"), ("turned", "turned", "turned")])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_linear_gradients_layouts(rows, k, n, lay, act):
    linear_gradient_case(rows, k, n, act=act, lay=lay)


def test_linear_gradient_of_float32_results():
    for act in ("none", "gelu_tanh"):
        linear_gradient_case(90, 136, 72, out="float32", grad="float32", act=act)


@pytest.mark.parametrize("what", [("dx",), ("dw",), ("dbias",), ("dw", "dbias"), ()])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_linear_gradients_asked_for(what, act):
    linear_gradient_case(70, 136, 264, act=act, what=what)


def test_linear_gradient_of_a_sum():
    """dy as the gradient of a sum over the results: one value, broadcast."""
    g = gen(5)
    x, w = U.matrix(g, 60, 72, "bfloat16"), U.matrix(g, 136, 72, "bfloat16", scale=0.1)
    dy = torch.ones((), dtype=torch.bfloat16, device="cuda").expand(60, 136)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    db = torch.empty(136, dtype=torch.bfloat16, device="cuda")
    for act in ("none", "silu"):
        with dpdr.Linear(60, 72, 136, act=act) as plan:
            plan.backward(x, w, dy, dx, dw, db)
            plan.sync()
        U.check_linear_gradients(x, w, None, dy, act, "bfloat16", "bfloat16", dx, dw, db)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("rows,k,n", GRAD_SIZES)
def test_gated_gradients(rows, k, n, keep):
    gated_gradient_case(rows, k, n, keep=keep)


def gated_gradient_case(rows, k, n, dtype="bfloat16", out=None, grad=None, act="silu", keep=False,
                        lay=("plain", "plain", "plain"), what=("dx", "dw")):
    g = gen(rows, k, n, 7)
    out, grad = out or dtype, grad or dtype
    x = U.matrix(g, rows, k, dtype, lay[0])
    wg, wu = (U.matrix(g, n, k, dtype, lay[1], k ** -0.5) for _ in range(2))
    dh = U.matrix(g, rows, n, out, lay[2])
    dx, dg, du = U.Guarded(rows, k, grad), U.Guarded(n, k, grad), U.Guarded(n, k, grad)
    ask = {}
    if "dx" in what:
        ask["dx"] = dx.t
    if "dw" in what:
        ask.update(dw_gate=dg.t, dw_up=du.t)
    with dpdr.Gated(rows + 2, k, n, dtype, out=out, grad=grad, act=act) as plan:
        pre = None
        if keep:
            pre = torch.empty(rows, 2 * n, device="cuda")
            plan.forward(x, wg, wu, torch.empty(rows, n, dtype=U.TYPES[out], device="cuda"), pre=pre)
        plan.backward(x, wg, wu, dh, pre=pre, **ask)
        plan.sync()
    U.check_gated_gradients(x, wg, wu, dh, act, dtype, grad, dx.check() if "dx" in what else None,
                            [dg.check(), du.check()] if "dw" in what else None)


@pytest.mark.parametrize("act", ACTS)
def test_gated_gradients_of_activations(act):
    gated_gradient_case(150, 200, 136, "float16", act=act)
    gated_gradient_case(150, 200, 136, out="float32", grad="float32", act=act, keep=True)


@pytest.mark.parametrize("rows,k,n", [(1, 72, 136), (20, 136, 72), (300, 264, 136)])
@pytest.mark.parametrize("lay", [("turned", "plain", "plain"), ("plain", "turned", "plain"), ("odd", "odd", "odd"),
                                 ("apart", "slack", "turned")])
def test_gated_gradients_layouts(rows, k, n, lay):
    gated_gradient_case(rows, k, n, lay=lay)


@pytest.mark.parametrize("what", [("dx",), ("dw",)])
def test_gated_gradients_asked_for(what):
    gated_gradient_case(70, 136, 264, what=what)


@pytest.mark.parametrize("act", ["gelu", "silu", "gelu_tanh"])
def test_gradients_against_differences(act):
    """The directional derivative of sum(dy * y) by central differences of the
    definition in 64 bits, against the kernels' gradients.  A step of 1e-4
    leaves 1e-8 of truncation; the gradients' own roundings (a relative
    2^-11 each, of random sign) stay below 2^-8 of the norms' product."""
    g = gen(11)
    rows, k, n = 37, 72, 136
    x, w, w2 = (U.matrix(g, r, k, "float16", scale=s) for r, s in ((rows, 1.0), (n, k ** -0.5), (n, k ** -0.5)))
    b = U.matrix(g, 1, n, "float16").reshape(-1)
    dy = U.matrix(g, rows, n, "float16")
    new = lambda t: torch.empty(t.shape, device="cuda")  # noqa: E731

    def compare(f, args, grads):
        for i, (a, d) in enumerate(zip(args, grads)):
            v = torch.randn(a.shape, generator=g).double().cuda()
            lo, hi = list(args), list(args)
            lo[i], hi[i] = a - 1e-4 * v, a + 1e-4 * v
            want = ((f(*hi) - f(*lo)) / 2e-4).item()
            got = (d.double() * v).sum().item()
            assert abs(got - want) <= 2.0 ** -8 * d.double().norm().item() + 1e-6, (i, got, want)

    d = [new(x), new(w), new(b)]
    with dpdr.Linear(rows, k, n, "float16", grad="float32", act=act) as plan:
        plan.backward(x, w, dy, d[0], d[1], d[2], bias=b)
        plan.sync()
    compare(lambda x, w, b: (dy.double() * U.act64(act, x @ w.t() + b)).sum(), [t.double() for t in (x, w, b)], d)
    d = [new(x), new(w), new(w2)]
    with dpdr.Gated(rows, k, n, "float16", grad="float32", act=act) as plan:
        plan.backward(x, w, w2, dy, d[0], d[1], d[2])
        plan.sync()
    compare(lambda x, w, w2: (dy.double() * U.act64(act, x @ w.t()) * (x @ w2.t())).sum(),
            [t.double() for t in (x, w, w2)], d)


@pytest.mark.parametrize("rows,k,n", [(2100, 2100, 2100), (1300, 1600, 3900), (2600, 2104, 1000), (2600, 1000, 2104)])
def test_products_whose_last_tiles_are_few(rows, k, n):
    """Sizes whose 256 x 256 tiles leave a last round of few, which is cut
    finer; twice on one plan, with the same bits."""
    g = gen(rows, k, n, 23)
    x, w, w2 = U.matrix(g, rows, k, "bfloat16"), *(U.matrix(g, n, k, "bfloat16", scale=k ** -0.5) for _ in range(2))
    dy = U.matrix(g, rows, n, "bfloat16")
    b = U.matrix(g, 1, n, "bfloat16").reshape(-1)
    with dpdr.Linear(rows, k, n, act="silu") as lin, dpdr.Gated(rows, k, n) as gat:
        first = None
        for _ in range(2):
            y, h, dx, dw, db = (torch.empty_like(t) for t in (dy, dy, x, w, b))
            gx, gg, gu = (torch.empty_like(t) for t in (x, w, w2))
            lin.forward(x, w, y, bias=b, residual=dy)
            lin.backward(x, w, dy, dx, dw, db, bias=b)
            gat.forward(x, w, w2, h)
            gat.backward(x, w, w2, dy, gx, gg, gu)
            lin.sync()
            gat.sync()
            got = [y, dx, dw, db, h, gx, gg, gu]
            assert first is None or all(torch.equal(p, q) for p, q in zip(first, got))
            first = got
    U.check_linear(y, x, w, b, dy, "silu", "bfloat16")
    U.check_linear_gradients(x, w, b, dy, "silu", "bfloat16", "bfloat16", dx, dw, db)
    U.check_gated(h, x, w, w2, "silu", "bfloat16")
    U.check_gated_gradients(x, w, w2, dy, "silu", "bfloat16", "bfloat16", gx, [gg, gu])


# ------------------------------------------------------- edges of the range

def test_no_rows():
    w = torch.randn(40, 24, device="cuda").to(torch.bfloat16)
    x, y = w.new_empty(0, 24), w.new_empty(0, 40)
    dw, dw2, db = torch.full_like(w, 3), torch.full_like(w, 3), torch.full_like(w[:, 0], 3)
    with dpdr.Linear(0, 24, 40) as plan:
        plan.forward(x, w, y)
        plan.backward(x, w, y, torch.empty_like(x), dw, db.contiguous())
        plan.sync()
        assert not dw.any()
    with dpdr.Linear(9, 24, 40, act="gelu") as plan:
        dw.fill_(3)
        db = torch.full((40,), 3, dtype=torch.bfloat16, device="cuda")
        plan.backward(x, w, y, torch.empty_like(x), dw, db)
        plan.sync()
        assert not dw.any() and not db.any()
    with dpdr.Gated(0, 24, 40) as plan:
        dw.fill_(3)
        plan.forward(x, w, w, y)
        plan.backward(x, w, w, y, torch.empty_like(x), dw, dw2)
        plan.sync()
        assert not dw.any() and not dw2.any()


@pytest.mark.parametrize("rows", [1, 20, 300])
@pytest.mark.parametrize("n", [40, 264])
def test_not_finite_values_stay_in_their_rows_and_columns(rows, n):
    """A NaN or infinity in row r of x or of w reaches row or column r of the
    result and nothing else, sizes that end inside a tile included."""
    k = 100
    g = gen(rows, n)
    x, w = U.matrix(g, rows, k, "bfloat16"), U.matrix(g, n, k, "bfloat16")
    x[rows - 1, k - 1] = float("nan")
    w[n - 1, 0] = float("inf")
    w[n // 2, k - 1] = float("nan")
    y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    with dpdr.Linear(rows, k, n) as plan:
        plan.forward(x, w, y)
        plan.sync()
    hit = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
    hit[rows - 1] = True
    hit[:, n - 1] = True
    hit[:, n // 2] = True
    assert torch.equal(~torch.isfinite(y), hit)
    want = x.double() @ w.double().t()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    h = torch.empty_like(y)
    with dpdr.Gated(rows, k, n, act="relu") as plan:
        plan.forward(x, w, w, h)
        plan.sync()
    assert torch.equal(torch.isnan(h), torch.isnan(U.act64("relu", want) * want))


def test_large_values_saturate():
    """Projections of +-1e4 and more: activations at their limits, no NaN."""
    x = torch.tensor([[3e4], [-3e4], [1e-3], [0.0]], device="cuda").to(torch.bfloat16)
    w = torch.ones(16, 1, dtype=torch.bfloat16, device="cuda")
    for act in ACTS:
        y, dx = torch.empty(4, 16, device="cuda"), torch.empty(4, 1, device="cuda")
        dy = torch.ones(4, 16, device="cuda")
        with dpdr.Linear(4, 1, 16, out="float32", grad="float32", act=act) as plan:
            plan.forward(x, w, y)
            plan.backward(x, w, dy, dx)
            plan.sync()
        U.check_linear(y, x, w, None, None, act, "float32")
        U.check_linear_gradients(x, w, None, dy, act, "bfloat16", "float32", dx)


def test_offsets_past_32_bits():
    """Rows of x, of the result and of the weights more than 2^31 elements
    into their arrays."""
    rows, k, n, pitch = 70_000, 64, 72, 32_768
    g = gen(13)
    base = torch.zeros(rows, pitch, dtype=torch.bfloat16, device="cuda")
    x = base[:, 64:64 + k]
    x.copy_(torch.randn(rows, k, generator=g).to(torch.bfloat16))
    w = U.matrix(g, n, k, "bfloat16", scale=0.125)
    y = base[:, 4096:4096 + n]
    dx = base[:, 8192:8192 + k]
    dw = torch.empty_like(w)
    with dpdr.Linear(rows, k, n) as plan:
        plan.forward(x, w, y)
        plan.sync()
        U.check_linear(y, x, w, None, None, "none", "bfloat16")
        plan.backward(x, w, y, dx, dw)
        plan.sync()
    U.check_linear_gradients(x, w, None, y, "none", "bfloat16", "bfloat16", dx, dw)
    wide = base[:, 64:64 + k]   # 70,000 weights, 32,768 apart, times a few rows
    few = U.matrix(g, 3, k, "bfloat16", scale=0.125)
    out = torch.empty(3, rows, dtype=torch.bfloat16, device="cuda")
    with dpdr.Linear(3, k, rows) as plan:
        plan.forward(few, wide, out)
        plan.sync()
    U.check_linear(out, few, wide, None, None, "none", "bfloat16")


def test_many_calls_of_one_plan_and_the_same_bits():
    """Calls of different row counts follow each other on one plan; the same
    call gives the same bits."""
    g = gen(17)
    k, n = 264, 520
    w, wu = (U.matrix(g, n, k, "bfloat16", scale=k ** -0.5) for _ in range(2))
    with dpdr.Linear(700, k, n, act="gelu") as lin, dpdr.Gated(700, k, n) as gat:
        first = {}
        for rows in (700, 1, 64, 333, 700, 17, 1, 64):
            x = U.matrix(gen(rows), rows, k, "bfloat16")
            dy = U.matrix(gen(rows, 1), rows, n, "bfloat16")
            y, h = torch.empty_like(dy), torch.empty_like(dy)
            r = [torch.empty_like(t) for t in (x, w, x, w, wu)]
            db = torch.empty(n, dtype=torch.bfloat16, device="cuda")
            lin.forward(x, w, y)
            gat.forward(x, w, wu, h)
            lin.backward(x, w, dy, r[0], r[1], db)
            gat.backward(x, w, wu, dy, r[2], r[3], r[4])
            got = [y, h, db] + r
            if rows in first:
                for a, b in zip(first[rows], got):
                    assert torch.equal(a, b)
            first[rows] = got
        lin.sync()
        gat.sync()
        U.check_linear(first[333][0], U.matrix(gen(333), 333, k, "bfloat16"), w, None, None, "gelu", "bfloat16")


def test_on_another_stream_and_in_a_graph():
    g = gen(19)
    rows, k, n = 130, 136, 264
    x, w = U.matrix(g, rows, k, "bfloat16"), U.matrix(g, n, k, "bfloat16", scale=0.1)
    y, dw, dx = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda"), torch.empty_like(w), torch.empty_like(x)
    side = torch.cuda.Stream()
    with dpdr.Linear(rows, k, n, act="silu") as plan:
        side.wait_stream(torch.cuda.current_stream())
        plan.forward(x, w, y, stream=side)
        plan.backward(x, w, y, dx, dw, stream=side)
        plan.sync(side)
        U.check_linear(y, x, w, None, None, "silu", "bfloat16")
        want = [t.clone() for t in (y, dx, dw)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.forward(x, w, y)
            plan.backward(x, w, y, dx, dw)
        for t in (y, dx, dw):
            t.zero_()
        graph.replay()
        graph.replay()
        plan.sync()
        for a, b in zip(want, (y, dx, dw)):
            assert torch.equal(a, b)


# ---------------------------------------------------------------- refusals

def test_refusals():
    mk = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    x, w, y = mk(4, 16), mk(24, 16), mk(4, 24)
    with dpdr.Linear(4, 16, 24) as plan, dpdr.Gated(4, 16, 24) as gated:
        for bad in (dict(x=mk(5, 16), y=mk(5, 24)), dict(w=mk(24, 15)), dict(y=mk(4, 23)),
                    dict(x=mk(4, 16, t=torch.float16)),
                    dict(y=mk(4, 24, t=torch.float32)), dict(bias=mk(23)), dict(bias=mk(48)[::2]),
                    dict(residual=mk(4, 24, t=torch.float32)), dict(pre=mk(4, 24)), dict(x=x.cpu()),
                    dict(y=mk(24, 4).t()), dict(y=mk(1, 24).expand(4, 24)), dict(x=mk(4, 16, 1))):
            a = dict(x=x, w=w, y=y)
            a.update(bad)
            with pytest.raises((dpdr.DpdrError, ValueError, TypeError)):
                plan.forward(a["x"], a["w"], a["y"], bias=a.get("bias"), residual=a.get("residual"), pre=a.get("pre"))
        # a result may not overlap an input or another result
        wide = mk(4, 64)
        with pytest.raises(dpdr.DpdrError):
            plan.forward(wide[:, :16], w, wide[:, 8:32])
        plan.forward(wide[:, :16], w, wide[:, 16:40])   # slices side by side do not
        with pytest.raises(dpdr.DpdrError):
            plan.forward(x, w, wide[:, 2:26], residual=wide[:, 1:25])
        with pytest.raises(dpdr.DpdrError):
            plan.backward(x, w, y, dx=x)
        d = mk(24, 16)
        with pytest.raises(dpdr.DpdrError):
            gated.backward(x, w, w, y, dw_gate=d, dw_up=d)
        with pytest.raises(dpdr.DpdrError):
            gated.backward(x, w, w, y, dw_gate=d)
        L = dpdr.lib()
        assert L.dpdr_linear(gated._h, 1, None, None, None, None, None, None, None) == dpdr.DPDR_ERR_INVALID
        assert L.dpdr_linear(plan._h, 1, None, None, None, None, None, None, None) == dpdr.DPDR_ERR_INVALID
        assert L.dpdr_gated(gated._h, -1, None, None, None, None, None, None) == dpdr.DPDR_ERR_INVALID
        odd = (ctypes.c_int64 * 3)(x.data_ptr() + 1, 16, 1)
        back = (ctypes.c_int64 * 3)(x.data_ptr(), -16, 1)
        ws = (ctypes.c_int64 * 3)(w.data_ptr(), 16, 1)
        ys = (ctypes.c_int64 * 3)(y.data_ptr(), 24, 1)
        for xs in (odd, back):
            assert L.dpdr_linear(plan._h, 3, xs, ws, None, None, ys, None, None) == dpdr.DPDR_ERR_INVALID
        plan.sync()
        gated.sync()
    for a in (("float32",), ("bfloat16", "float16"), ("bfloat16", None, "int32"), ("bfloat16", None, None, "tanh")):
        with pytest.raises((ValueError, dpdr.DpdrError)):
            dpdr.Linear(4, 4, 4, *a)
    for a in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (1 << 31, 4, 4)):
        with pytest.raises(dpdr.DpdrError):
            dpdr.Gated(*a)


# ----------------------------------------------------------- in use together

@pytest.mark.parametrize("ranks,rows,model,hidden", [(4, 200, 264, 544), (1, 1, 64, 128), (7, 33, 136, 700),
                                                     (2, 600, 512, 2048)])
def test_feed_forward_split_over_ranks(ranks, rows, model, hidden):
    """The example: Gated, Linear with float32 partials, and the all-reduce,
    forward and backward, against the whole block in 64 bits.  Roundings to
    bfloat16 on the way of a result, 2^-9 of the norm each: h for y and
    dw_down; dy or dh and then dg and du for the others (2, 3 and the
    gradient of the activation from a float32 projection)."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import tensor_parallel_ffn as ffn
    block = ffn.SplitFeedForward(ranks, rows, model, hidden)
    g = gen(29, ranks)
    x = U.matrix(g, rows, model, "bfloat16")
    dy = U.matrix(g, rows, model, "float32")
    ys = block.forward(x)
    dxs = block.backward(x, dy)
    block.sync()
    for copies in (ys, dxs):   # every rank holds the same bits
        assert all(torch.equal(copies[0], c) for c in copies)
    errors = ffn.worst(block, x, dy)
    for name, steps in (("y", 1), ("dw_down", 2), ("dx", 3), ("dw_gate", 3), ("dw_up", 3)):
        assert errors[name] <= steps * 2.0 ** -8, (name, errors)
    block.close()
