"""The experts' host code over a CUDA runtime that only keeps books: a row of what the
products read by whole pieces of weights holds all of its last piece, so that no piece
reaches into the next row's values."""
import ctypes
import os
import subprocess

import pytest

from paper_2109_12626_gb300 import _native as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")
BF16, F16, I8 = N.DPDR_BFLOAT16, N.DPDR_FLOAT16, N.DPDR_INT8


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("fake") / "experts_rows_fake.so")
    csrc = os.path.join(ROOT, "paper_2109_12626_gb300", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fPIC", "-shared", "-I", os.path.join(CUDA, "include"),
                        "-I", csrc, "-I", os.path.join(ROOT, "tests"), os.path.join(csrc, "proj.cpp"),
                        os.path.join(csrc, "experts.cpp"), os.path.join(ROOT, "tests", "experts_rows_fake.cpp"), "-o", so,
                        "-Wl,-z,defs", "-Wl,-Bsymbolic", "-lpthread"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    L = ctypes.CDLL(so)
    for name, (res, args) in N.SIGNATURES.items():
        if name.startswith("dpdr_experts"):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
    L.fake_d_pad.restype = L.fake_h_pad.restype = ctypes.c_long
    L.fake_wrong.restype = L.fake_message.restype = ctypes.c_char_p
    return L


# elements of a piece of weights, at most: 128 bytes of 8-bit weights in the gate and up
# products, 64 in the down products, 64 or 128 bytes of 16-bit ones
@pytest.mark.parametrize("weights,up,down", [(BF16, 64, 64), (F16, 64, 64), (I8, 128, 64)])
@pytest.mark.parametrize("d,h", [(1, 1), (64, 64), (65, 63), (128, 64), (129, 100), (192, 320), (2880, 1000), (4096, 1792)])
def test_a_piece_stays_in_its_row(fake, weights, up, down, d, h):
    operands = F16 if weights == F16 else BF16
    plan = fake.dpdr_experts_plan(3, d, h, 4, 2, 0, 4, operands, weights, operands, 4, 1)
    assert plan, fake.fake_message()
    held = [(ctypes.c_int64 * n)(*v) for n, v in ((3, (1 << 20, d, 1)), (3, (1 << 24, d, 1)), (4, (1 << 32, h * d, d, 1)),
                                                  (4, (1 << 36, h * d, d, 1)), (4, (1 << 40, d * h, h, 1)), (3, (1 << 28, d, 1)))]
    x, router, gate, up_, w_down, y = (ctypes.addressof(m) for m in held)
    scale = [1 << 41, 1 << 42, 1 << 43] if weights == I8 else [None] * 3
    assert fake.dpdr_experts(plan, 3, x, router, gate, up_, w_down, *scale, y, None, None, None) == 0, fake.fake_message()
    assert fake.fake_wrong() == b""
    assert (d + up - 1) // up * up <= fake.fake_d_pad()
    assert (h + down - 1) // down * down <= fake.fake_h_pad()
    fake.dpdr_experts_destroy(plan)
