"""The kernel of 256 x 256 tiles with everything that a finished sum may need:
the sizes are derived from the SMs, so that few-row kernels do not take them
(test_projections_fake.py checks which kernel does)."""
import pytest
import torch

import paper_2109_12626_gb300 as dpdr
import proj_util as U
import test_gpu_projections as T
from proj_tiles import tile_size

pytestmark = pytest.mark.gpu


def size(odd=0):
    rows, n = tile_size(torch.cuda.get_device_properties(0).multi_processor_count)
    return rows, n + odd


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("act", T.ACTS)
def test_activations_and_kept_projections(act, dtype, odd):
    rows, n = size(odd)
    T.linear_case(rows, 264, n, dtype, act=act, pre=True)
    T.linear_case(rows, 264, n, dtype, act=act, out="float32", pre=True, residual=odd == 0)
    T.gated_case(rows, 264, n, dtype, act=act, pre=True)
    T.gated_case(rows, 264, n, dtype, act=act, out="float32", pre=True)


@pytest.mark.parametrize("k", [640, 641, 1300, 2500])
@pytest.mark.parametrize("odd", [0, 1])
def test_float32_results_of_several_runs(k, odd):
    rows, n = size(odd)
    T.linear_case(rows, k, n, act="gelu", out="float32")
    T.gated_case(rows, k, n, out="float32")


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("lx", ["plain", "turned", "slack", "odd", "apart"])
@pytest.mark.parametrize("lw", ["plain", "turned", "slack", "odd", "apart"])
def test_layouts(lx, lw, out):
    rows, n = size()
    T.linear_case(rows, 250, n, lay=(lx, lw), out=out)
    T.gated_case(rows, 250, n, lay=(lx, lw, lw), out=out)


@pytest.mark.parametrize("out", ["float16", "float32"])
@pytest.mark.parametrize("guard", [(1, 2), (2, 2), (4, 5), (3, 0), (8, 8)])
@pytest.mark.parametrize("odd", [0, 2, 3])
def test_result_places(out, guard, odd):
    rows, n = size(odd)
    T.linear_case(rows, 72, n, "float16", out=out, guard=guard, act="relu")
    T.gated_case(rows, 72, n, "float16", out=out, guard=guard)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_onto_the_residual(out, odd, act):
    rows, n = size(odd)
    g = T.gen(rows, n, 1)
    x, w = U.matrix(g, rows, 136, "bfloat16"), U.matrix(g, n, 136, "bfloat16", scale=136 ** -0.5)
    y = U.Guarded(rows, n, out)
    r = U.matrix(g, rows, n, out)
    y.t.copy_(r)
    with dpdr.Linear(rows, 136, n, "bfloat16", out=out, act=act) as plan:
        plan.forward(x, w, y.t, residual=y.t)
        plan.sync()
    U.check_linear(y.check(), x, w, None, r, act, out)


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_residual_as_broadcast_and_turned(out):
    rows, n = size()
    g = T.gen(9, rows)
    x, w = U.matrix(g, rows, 64, "bfloat16"), U.matrix(g, n, 64, "bfloat16", scale=0.125)
    y = torch.empty(rows, n, dtype=U.TYPES[out], device="cuda")
    for r in (U.matrix(g, 1, n, out).expand(rows, n), U.matrix(g, rows, 1, out).expand(rows, n),
              U.matrix(g, rows, n, out, "turned"), U.matrix(g, rows, n, out, "odd")):
        with dpdr.Linear(rows, 64, n, out=out) as plan:
            plan.forward(x, w, y, residual=r)
            plan.sync()
        U.check_linear(y, x, w, None, r, "none", out)


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("act", T.ACTS)
def test_gradients(act, odd, monkeypatch):
    """Computed again and kept, 16-bit and float32 gradients and results; dx
    and dw are products of tiles too.  The slope of relu jumps at 0, and of
    1.6 million z one or two lie within their error of it: a dz that is there
    or not is 1e-3 of the norm, which the bound of each element allows for and
    that of the norm does not."""
    rows, n = size(odd)
    if act == "relu":
        monkeypatch.setattr(U, "close_in_norm", lambda *a: None)
    for keep in (False, True):
        T.linear_gradient_case(rows, n, n + 4, "float16", grad="float32", act=act, keep=keep)
        T.gated_gradient_case(rows, n, n + 4, act=act, keep=keep)
    T.gated_gradient_case(rows, n, n, "float16", out="float32", grad="float32", act=act)


def test_not_finite_values_stay_in_their_rows_and_columns():
    rows, n = size(1)
    g = T.gen(rows, n)
    x, w = U.matrix(g, rows, 100, "bfloat16"), U.matrix(g, n, 100, "bfloat16")
    x[rows - 1, 99] = float("nan")
    w[n - 1, 0] = float("inf")
    w[n // 2, 99] = float("nan")
    hit = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
    hit[rows - 1] = True
    hit[:, n - 1] = True
    hit[:, n // 2] = True
    want = x.double() @ w.double().t()
    for out in ("bfloat16", "float32"):
        y = torch.empty(rows, n, dtype=U.TYPES[out], device="cuda")
        with dpdr.Linear(rows, 100, n, out=out) as plan:
            plan.forward(x, w, y)
            plan.sync()
        assert torch.equal(~torch.isfinite(y), hit)
        assert torch.equal(torch.isnan(y), torch.isnan(want))
