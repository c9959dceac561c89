"""Projection plans in use: captured calls among others, and what a plan's
failures leave behind."""
import pytest
import torch

import paper_2109_12626_gb300 as dpdr
import proj_util as U

pytestmark = pytest.mark.gpu


def gen(*key):
    return torch.Generator().manual_seed(hash(key) % (1 << 31))


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("rows,k,n", [(33, 100, 70), (700, 250, 1001)])
def test_a_captured_call_is_replayed_after_others(rows, k, n, act):
    """A graph of calls that copy operands and use scratch, replayed after
    calls of every other kind on the same plan: other ways round, with the
    bias gradient, more rows."""
    g = gen(rows, k, n, act == "silu")
    new = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x, w = U.matrix(g, rows, k, "bfloat16", "odd"), U.matrix(g, n, k, "bfloat16", "odd", k ** -0.5)
    dy = U.matrix(g, rows, n, "bfloat16", "odd")
    y, dx, dw = new(rows, n), new(rows, k), new(n, k)
    with dpdr.Linear(3 * rows, k, n, act=act) as plan:
        def call():
            plan.forward(x, w, y)
            plan.backward(x, w, dy, dx, dw)
        call()   # makes the scratch
        plan.sync()
        want = [t.clone() for t in (y, dx, dw)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for m in (3 * rows, 1, rows):
            for how in ("turned", "apart", "odd", "plain"):
                x2, w2 = U.matrix(g, m, k, "bfloat16", how), U.matrix(g, n, k, "bfloat16", how)
                dy2 = U.matrix(g, m, n, "bfloat16", how)
                plan.forward(x2, w2, new(m, n))
                plan.backward(x2, w2, dy2, new(m, k), new(n, k), new(n))
        plan.sync()
        others = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]
        for t in (y, dx, dw):
            t.zero_()
        graph.replay()
        plan.sync()
        for a, b in zip(want, (y, dx, dw)):
            assert torch.equal(a, b)
        assert all(bool((t == 3.0).all()) for t in others)


def test_scratch_that_does_not_fit_is_forgotten():
    """A call whose scratch does not fit fails; the plan and the library's
    other entry points go on as before."""
    import ctypes
    import paper_2109_12626_gb300._native as N
    g = gen(41)
    x, w, dy = U.matrix(g, 4, 16, "bfloat16"), U.matrix(g, 8192, 16, "bfloat16"), U.matrix(g, 4, 8192, "bfloat16")
    dx, y = torch.empty_like(x), torch.empty_like(dy)
    a = torch.arange(100, dtype=torch.int32, device="cuda")
    b = torch.empty_like(a)
    with dpdr.Linear((1 << 31) - 1, 16, 8192, act="silu") as plan:
        for _ in range(2):   # 35 TB of dz
            with pytest.raises(dpdr.DpdrError) as e:
                plan.backward(x, w, dy, dx)
            assert e.value.status == N.DPDR_ERR_OOM
            one = (ctypes.c_void_p * 1)
            rc = N.lib().dpdr_allreduce_schedule_noalloc(1, 100, N.DPDR_INT32, N.DPDR_OP_SUM, 1, one(a.data_ptr()),
                                                         one(b.data_ptr()), torch.cuda.current_stream().cuda_stream)
            assert rc == N.DPDR_OK, N.lib().dpdr_last_error_message()
            assert torch.equal(a, b)
        plan.forward(x, w, y)
        plan.sync()
    U.check_linear(y, x, w, None, None, "silu", "bfloat16")
