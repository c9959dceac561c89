"""The host code of the 8-bit products and the experts over a CUDA runtime that
only keeps books (serving_fake.cpp): scratch, devices, refusals, which kernels a
call takes."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2109_12626_gb300 import _native as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")
BF16, F16, F32, I8 = N.DPDR_BFLOAT16, N.DPDR_FLOAT16, N.DPDR_FLOAT32, N.DPDR_INT8


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    # -Bsymbolic: its own CUDA runtime, not one that the process already has
    so = str(tmp_path_factory.mktemp("fake") / "serving_fake.so")
    csrc = os.path.join(ROOT, "paper_2109_12626_gb300", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fPIC", "-shared", "-I", os.path.join(CUDA, "include"),
                        "-I", csrc, "-I", os.path.join(ROOT, "tests"), os.path.join(csrc, "proj.cpp"),
                        os.path.join(csrc, "integer.cpp"), os.path.join(csrc, "experts.cpp"),
                        os.path.join(ROOT, "tests", "serving_fake.cpp"), "-o", so, "-Wl,-z,defs", "-Wl,-Bsymbolic",
                        "-lpthread"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    L = ctypes.CDLL(so)
    for name, (res, args) in N.SIGNATURES.items():
        if name.startswith(("dpdr_integer", "dpdr_experts", "dpdr_quantise")):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
    for name in ("fake_frees", "fake_launches", "fake_streamed", "fake_widened", "fake_layers", "fake_copies", "fake_tiles"):
        getattr(L, name).restype = ctypes.c_long
    L.fake_wrong.restype = L.fake_message.restype = ctypes.c_char_p
    return L


@pytest.fixture
def fake(built):
    built.fake_reset()
    built.fake_counts_reset()
    return built


class Arrays:
    """A caller's arrays: addresses that nothing reads, one region each."""

    def __init__(self):
        self.at, self.held = 1 << 30, []

    def place(self, size, off=0):
        p = self.at + off
        self.at += (size + off + 511) // 256 * 256
        return p

    def matrix(self, rows, cols, how="plain", esize=1):
        rs, cs, off = {"plain": (cols, 1, 0), "turned": (1, rows, 0), "slack": ((cols + 63) // 64 * 64, 1, 0),
                       "odd": (cols + 3, 1, 1), "apart": (2 * cols, 2, 0), "broadcast": (0, 1, 0)}[how]
        m = (ctypes.c_int64 * 3)(self.place((rows * max(rs, 1) + cols * max(cs, 1) + 16) * esize, off * esize), rs, cs)
        self.held.append(m)
        return ctypes.addressof(m)

    def stack(self, count, rows, cols, esize, pad=0, cs=1):
        rs = cols + pad
        m = (ctypes.c_int64 * 4)(self.place((count * rows * rs + 64) * esize), rows * rs, rs, cs)
        self.held.append(m)
        return ctypes.addressof(m)

    def vector(self, n):
        return self.place(4 * n + 4)


LAYOUTS = ["plain", "turned", "slack", "odd", "apart", "broadcast"]


@pytest.mark.parametrize("out", [BF16, F16, F32])
@pytest.mark.parametrize("most,k,n", [(1, 13, 9), (5, 64, 300), (64, 100, 37), (333, 24, 130), (5000, 70, 8), (9, 700, 1),
                                      (200, 1, 50), (700, 2000, 20000)])
def test_integer_scratch_never_moves(fake, out, most, k, n):
    """Whatever calls follow each other on a plan, nothing that an earlier one used
    is freed before the plan is, and every place that a kernel gets holds what it
    reads and writes there."""
    r = random.Random(most * 7 + out)
    for _ in range(20):
        plan = fake.dpdr_integer_plan(most, k, n, out)
        assert plan
        for _ in range(12):
            a, rows, es = Arrays(), r.choice([0, 1, most, r.randint(0, most), min(most, 4)]), 4 if out == F32 else 2
            maybe = lambda v: v if r.random() < 0.5 else None  # noqa: E731
            rc = fake.dpdr_integer_linear(plan, rows, a.matrix(rows, k, r.choice(LAYOUTS)), a.vector(rows),
                                          a.matrix(n, k, r.choice(LAYOUTS)), a.vector(n), maybe(a.vector(n)),
                                          maybe(a.matrix(rows, n, r.choice(LAYOUTS), es)), a.matrix(rows, n, "plain", es), None)
            assert rc == 0, fake.fake_message()
            assert fake.fake_frees() == 0 and fake.fake_wrong() == b""
        fake.dpdr_integer_destroy(plan)
        assert fake.fake_live() == 0
        fake.fake_reset()


@pytest.mark.parametrize("most", [1, 7, 8, 9, 16, 17, 64])
@pytest.mark.parametrize("operands,weights,result", [(BF16, BF16, BF16), (F16, F16, F32), (BF16, I8, F32), (F16, I8, F16),
                                                     (BF16, BF16, F32), (F16, F16, F16)])
@pytest.mark.parametrize("d,h,experts,top,first,local", [(1, 1, 1, 1, 0, 1), (100, 37, 8, 2, 0, 8), (64, 2000, 512, 16, 100, 3),
                                                         (4096, 1024, 64, 8, 32, 32), (33, 16, 40, 3, 39, 1)])
def test_experts_scratch(fake, most, operands, weights, result, d, h, experts, top, first, local):
    plan = fake.dpdr_experts_plan(most, d, h, experts, top, first, local, operands, weights, result, 4, 1)
    assert plan, fake.fake_message()
    es, os_ = (1 if weights == I8 else 2), (4 if result == F32 else 2)
    for rows in (most, 0, 1, most // 2, most):
        a = Arrays()
        scale = [a.vector(local * h), a.vector(local * h), a.vector(local * d)] if weights == I8 else [None] * 3
        rc = fake.dpdr_experts(plan, rows, a.matrix(rows, d, "odd", 2), a.matrix(experts, d, "turned", 2),
                               a.stack(local, h, d, es), a.stack(local, h, d, es, 3), a.stack(local, d, h, es), *scale,
                               a.matrix(rows, d, "slack", os_), a.vector(rows * top), a.vector(rows * top), None)
        assert rc == 0, fake.fake_message()
    assert fake.fake_layers() == (4 if most > 1 else 3)
    assert fake.fake_wrong() == b"" and fake.fake_frees() == 0
    fake.dpdr_experts_destroy(plan)
    assert fake.fake_live() == 0


def test_pieces_are_counted_in_32_bits(fake):
    """Weights that no memory holds (or one matrix for many experts) whose pieces
    pass 2^30 are refused."""
    assert not fake.dpdr_experts_plan(64, 1 << 20, 1 << 20, 512, 16, 0, 512, BF16, BF16, BF16, 4, 1)
    assert b"pieces" in fake.fake_message()
    assert fake.fake_live() == 0


def test_which_kernel_a_product_takes(fake):
    a = Arrays()
    plan = fake.dpdr_integer_plan(9000, 256, 512, BF16)

    def call(rows, how_x="plain", how_w="plain"):
        fake.fake_counts_reset()
        before = fake.fake_tiles()
        assert fake.dpdr_integer_linear(plan, rows, a.matrix(rows, 256, how_x), a.vector(rows), a.matrix(512, 256, how_w),
                                        a.vector(512), None, None, a.matrix(rows, 512, "plain", 2), None) == 0
        return fake.fake_streamed(), fake.fake_widened(), fake.fake_tiles() - before, fake.fake_copies()

    assert call(1) == call(16) == (1, 0, 0, 0)
    assert call(3, "odd") == call(16, "turned") == (1, 0, 0, 1)
    assert call(1, "odd", "odd") == call(2, "odd", "odd") == (1, 0, 0, 0)
    assert call(3, "odd", "odd") == (1, 0, 0, 1)
    assert call(17) == call(200) == call(40, "odd", "odd") == (0, 1, 0, 0)
    assert call(9000) == call(5, "plain", "turned") == call(100, "turned") == (0, 0, 1, 1)
    fake.dpdr_integer_destroy(plan)


def test_calls_on_another_device_are_refused(fake):
    a = Arrays()
    fake.fake_device(1)
    lin = fake.dpdr_integer_plan(4, 64, 32, BF16)
    moe = fake.dpdr_experts_plan(4, 64, 32, 4, 2, 0, 4, BF16, BF16, BF16, 4, 1)
    x, y = a.matrix(4, 64, "plain", 2), a.matrix(4, 64, "plain", 2)
    calls = [lambda: fake.dpdr_integer_linear(lin, 4, a.matrix(4, 64), a.vector(4), a.matrix(32, 64), a.vector(32), None, None,
                                              a.matrix(4, 32, "plain", 2), None),
             lambda: fake.dpdr_experts(moe, 4, x, a.matrix(4, 64, "plain", 2), a.stack(4, 32, 64, 2), a.stack(4, 32, 64, 2),
                                       a.stack(4, 64, 32, 2), None, None, None, y, None, None, None)]
    for device, rc in ((0, N.DPDR_ERR_INVALID), (2, N.DPDR_ERR_INVALID), (1, N.DPDR_OK)):
        fake.fake_device(device)
        before = fake.fake_launches()
        for call in calls:
            assert call() == rc
            assert rc == N.DPDR_OK or b"device" in fake.fake_message()
        assert (fake.fake_launches() > before) == (rc == N.DPDR_OK)
    fake.dpdr_integer_destroy(lin)
    fake.dpdr_experts_destroy(moe)


@pytest.mark.parametrize("what", ["rows", "x", "router", "gate turned", "down NULL", "stack stride", "far", "y turned", "y over x",
                                  "chosen over y", "scale", "share over chosen", "w odd"])
def test_experts_calls_refused(fake, what):
    a = Arrays()
    plan = fake.dpdr_experts_plan(4, 64, 32, 4, 2, 0, 4, BF16, BF16, BF16, 4, 1)
    args = dict(x=a.matrix(4, 64, "plain", 2), router=a.matrix(4, 64, "plain", 2), gate=a.stack(4, 32, 64, 2),
                up=a.stack(4, 32, 64, 2), down=a.stack(4, 64, 32, 2), gs=None, us=None, ds=None,
                y=a.matrix(4, 64, "plain", 2), chosen=a.vector(8), share=a.vector(8))
    rows = 4

    def stack(at, *strides):
        m = (ctypes.c_int64 * 4)(at, *strides)
        a.held.append(m)
        return ctypes.addressof(m)

    if what == "rows":
        rows = 5
    elif what in ("x", "router"):
        args[what] = None
    elif what == "gate turned":
        args["gate"] = a.stack(4, 32, 64, 2, 0, 32)
    elif what == "down NULL":
        args["down"] = None
    elif what == "stack stride":
        args["up"] = stack(1 << 40, -64, 64, 1)
    elif what == "far":
        args["up"] = stack(1 << 40, 64, 1 << 58, 1)
    elif what == "w odd":
        args["up"] = stack((1 << 40) + 1, 2048, 64, 1)
    elif what == "y turned":
        args["y"] = a.matrix(4, 64, "turned", 2)
    elif what == "y over x":
        args["y"] = args["x"]
    elif what == "chosen over y":
        args["chosen"] = ctypes.cast(args["y"], ctypes.POINTER(ctypes.c_int64))[0] + 16
    elif what == "scale":
        args["us"] = a.vector(4 * 32)
    elif what == "share over chosen":
        args["share"] = args["chosen"] + 16
    assert fake.dpdr_experts(plan, rows, *args.values(), None) == N.DPDR_ERR_INVALID
    assert b"dpdr_experts" in fake.fake_message() and fake.fake_layers() == 0
    fake.dpdr_experts_destroy(plan)


def test_memory_that_runs_out(fake):
    """An allocation that fails is told, and leaves plans that can be called again."""
    a = Arrays()
    lin = fake.dpdr_integer_plan(300, 70, 40000, BF16)
    args = lambda rows: (a.matrix(rows, 70, "odd"), a.vector(rows), a.matrix(40000, 70), a.vector(40000), None, None,  # noqa: E731
                         a.matrix(rows, 40000, "plain", 2), None)
    for rows in (3, 300):
        for fails in (1, 1):
            fake.fake_refuse_mallocs(fails)
            assert fake.dpdr_integer_linear(lin, rows, *args(rows)) == N.DPDR_ERR_OOM
        assert fake.dpdr_integer_linear(lin, rows, *args(rows)) == 0
    fake.dpdr_integer_destroy(lin)
    fake.fake_refuse_mallocs(1)
    assert not fake.dpdr_experts_plan(4, 64, 32, 4, 2, 0, 4, BF16, BF16, BF16, 4, 1)
    lived = fake.fake_live()
    fake.fake_refuse_mallocs(1)
    assert not fake.dpdr_integer_plan(4, 64, 32, BF16)
    fake.fake_refuse_mallocs(0)
    assert fake.fake_live() == lived
    assert fake.fake_live() == 0 and fake.fake_wrong() == b""
