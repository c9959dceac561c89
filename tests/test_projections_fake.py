"""The projections' host code over a CUDA runtime that only keeps books
(proj_fake.cpp): allocations, devices and errors of plans and calls."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2109_12626_gb300 import _native as N
from proj_tiles import tile_size

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")
BF16, F16, F32 = N.DPDR_BFLOAT16, N.DPDR_FLOAT16, N.DPDR_FLOAT32


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    # -Bsymbolic: its own CUDA runtime, not one that the process already has
    so = str(tmp_path_factory.mktemp("fake") / "proj_fake.so")
    csrc = os.path.join(ROOT, "paper_2109_12626_gb300", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fPIC", "-shared", "-I", os.path.join(CUDA, "include"),
                        "-I", csrc, os.path.join(csrc, "proj.cpp"), os.path.join(ROOT, "tests", "proj_fake.cpp"),
                        "-o", so, "-Wl,-z,defs", "-Wl,-Bsymbolic", "-lpthread"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    L = ctypes.CDLL(so)
    for name, (res, args) in N.SIGNATURES.items():
        if name.startswith(("dpdr_linear", "dpdr_gated", "dpdr_proj")):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
    for name in ("fake_frees", "fake_launches", "fake_syncs", "fake_tiles", "fake_rows"):
        getattr(L, name).restype = ctypes.c_long
    L.fake_wrong.restype = L.fake_message.restype = ctypes.c_char_p
    return L


@pytest.fixture
def fake(built):
    built.fake_reset()
    return built


class Arrays:
    """Matrices of a caller: addresses that nothing reads, one region each."""

    def __init__(self):
        self.at, self.held = 1 << 30, []

    def matrix(self, rows, cols, how="plain", esize=2):
        rs, cs, off = {"plain": (cols, 1, 0), "turned": (1, rows, 0), "slack": ((cols + 15) // 8 * 8, 1, 0),
                       "odd": (cols + 3, 1, 1), "apart": (2 * cols, 2, 0), "broadcast": (0, 1, 0)}[how]
        m = (ctypes.c_int64 * 3)(self.at + off * esize, rs, cs)
        self.at += ((rows * max(rs, 1) + cols * max(cs, 1) + 16) * 8 + 255) // 256 * 256
        self.held.append(m)
        return ctypes.addressof(m)

    def vector(self, n):
        self.at += (8 * n + 255) // 256 * 256
        return self.at - (8 * n + 255) // 256 * 256


LAYOUTS = ["plain", "turned", "slack", "odd", "apart"]


def random_call(L, plan, gated, r, rows, k, n, out, grad):
    """One forward or backward call of random layouts; its status."""
    a, es, qs = Arrays(), 4 if out == F32 else 2, 4 if grad == F32 else 2
    how = lambda: r.choice(LAYOUTS)  # noqa: E731
    x, w = a.matrix(rows, k, how()), [a.matrix(n, k, how()) for _ in range(2)]
    maybe = lambda v: v if r.random() < 0.5 else None  # noqa: E731
    if r.random() < 0.4:
        y = a.matrix(rows, n, "plain", es)
        if gated:
            return L.dpdr_gated(plan, rows, x, w[0], w[1], y, maybe(a.matrix(rows, 2 * n, "plain", 4)), None)
        return L.dpdr_linear(plan, rows, x, w[0], maybe(a.vector(n)), maybe(a.matrix(rows, n, how(), es)), y,
                             maybe(a.matrix(rows, n, "plain", 4)), None)
    dy = a.matrix(rows, n, r.choice(LAYOUTS + ["broadcast"]), es)
    dx = maybe(a.matrix(rows, k, "plain", qs))
    dw = [a.matrix(n, k, "plain", qs) for _ in range(2)]
    if gated:
        dw = dw if r.random() < 0.5 else [None, None]
        return L.dpdr_gated_backward(plan, rows, x, w[0], w[1], dy, maybe(a.matrix(rows, 2 * n, "plain", 4)), dx,
                                     dw[0], dw[1], None)
    return L.dpdr_linear_backward(plan, rows, x, w[0], maybe(a.vector(n)), dy, maybe(a.matrix(rows, n, "plain", 4)),
                                  dx, maybe(dw[0]), maybe(a.vector(n)), None)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", [0, 4])
@pytest.mark.parametrize("out,grad", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("most,k,n", [(1, 13, 9), (60, 100, 37), (333, 24, 130), (5000, 70, 8), (9, 700, 1)])
def test_scratch_never_moves(fake, gated, act, out, grad, most, k, n):
    """Whatever calls follow each other on a plan, in any order, nothing that
    an earlier one used is freed before the plan is (a captured call may be
    replayed), and every place that a kernel gets holds what it writes."""
    r = random.Random(most * 7 + act)
    make = fake.dpdr_gated_plan if gated else fake.dpdr_linear_plan
    for _ in range(20):
        plan = make(most, k, n, BF16, out, grad, act)
        assert plan
        for _ in range(12):
            rows = r.choice([0, 1, most, r.randint(0, most)])
            assert random_call(fake, plan, gated, r, rows, k, n, out, grad) == 0, fake.fake_message()
            assert fake.fake_frees() == 0
            assert fake.fake_wrong() == b""
        fake.dpdr_proj_destroy(plan)
        assert fake.fake_live() == 0
        fake.fake_reset()


def test_calls_on_another_device_are_refused(fake):
    """A plan's scratch and arrays lie on its device: with another one
    current, a call launches nothing."""
    a = Arrays()
    x, w, y, d = a.matrix(4, 16), a.matrix(24, 16), a.matrix(4, 24), a.matrix(4, 16)
    fake.fake_device(1)
    lin, gat = fake.dpdr_linear_plan(4, 16, 24, BF16, BF16, BF16, 4), fake.dpdr_gated_plan(4, 16, 24, BF16, BF16, BF16, 4)
    calls = [lambda: fake.dpdr_linear(lin, 4, x, w, None, None, y, None, None),
             lambda: fake.dpdr_gated(gat, 4, x, w, w, y, None, None),
             lambda: fake.dpdr_linear_backward(lin, 4, x, w, None, y, None, d, None, None, None),
             lambda: fake.dpdr_gated_backward(gat, 4, x, w, w, y, None, d, None, None, None)]
    for device, rc in ((0, N.DPDR_ERR_INVALID), (2, N.DPDR_ERR_INVALID), (1, N.DPDR_OK)):
        fake.fake_device(device)
        before = fake.fake_launches()
        for call in calls:
            assert call() == rc
            assert rc == N.DPDR_OK or b"device" in fake.fake_message()
        assert (fake.fake_launches() > before) == (rc == N.DPDR_OK)
    fake.dpdr_proj_destroy(lin)
    fake.dpdr_proj_destroy(gat)


def test_many_plans_at_a_time(fake):
    """As many plans as there is memory for, each with an error word of its
    own; those given back are taken again."""
    plans = [fake.dpdr_linear_plan(1, 8, 8, BF16, BF16, BF16, 0) for _ in range(20000)]
    assert all(plans), fake.fake_message()
    for p in plans[::3]:
        fake.dpdr_proj_destroy(p)
    plans[::3] = [fake.dpdr_linear_plan(1, 8, 8, BF16, BF16, BF16, 0) for _ in plans[::3]]
    assert all(plans)
    words = fake.fake_error_words((ctypes.c_void_p * len(plans))(*plans), len(plans))
    assert words == len(plans)
    for p in plans:
        fake.dpdr_proj_destroy(p)


@pytest.mark.parametrize("most", [10, 128, 256, 512])
def test_runs_of_a_sum(fake, most):
    """Sums of up to 2^31 elements (2^25 steps of 64; of two chained ones
    2^26) split into runs: none empty or too long, every step in one."""
    for steps in [*range(1, 200), 999, 146540, 146541, 160000, (1 << 25) - 1, 1 << 25, 1 << 26]:
        assert fake.fake_runs_fit(steps, most), steps


def test_which_kernel_the_tile_tests_reach(fake):
    """The sizes of test_gpu_projections_tiles.py (on this many SMs, which the
    fake reports) go to the kernel of tiles: forward, dx and dw."""
    a = Arrays()
    rows, n = tile_size(152)
    for odd in (0, 1, 2, 3):
        for k in (64, 264, 2500, n):
            x, w = a.matrix(rows, k), [a.matrix(n + odd, k) for _ in range(2)]
            y, dx, dw = a.matrix(rows, n + odd), a.matrix(rows, k), [a.matrix(n + odd, k) for _ in range(2)]
            lin, gat = fake.dpdr_linear_plan(rows, k, n + odd, BF16, BF16, BF16, 4), \
                fake.dpdr_gated_plan(rows, k, n + odd, BF16, BF16, BF16, 4)
            assert fake.dpdr_linear(lin, rows, x, w[0], None, None, y, None, None) == 0
            assert fake.dpdr_gated(gat, rows, x, w[0], w[1], y, None, None) == 0
            assert (fake.fake_tiles(), fake.fake_rows()) == (2, 0)
            if k == n:
                assert fake.dpdr_linear_backward(lin, rows, x, w[0], None, y, None, dx, dw[0], None, None) == 0
                assert fake.dpdr_gated_backward(gat, rows, x, w[0], w[1], y, None, dx, dw[0], dw[1], None) == 0
                assert (fake.fake_tiles(), fake.fake_rows()) == (8, 0)
            fake.dpdr_proj_destroy(lin)
            fake.dpdr_proj_destroy(gat)
            fake.fake_reset()
