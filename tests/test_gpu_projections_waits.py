"""The bounded waits of the projections' kernels: one that runs out says so to
its whole warp and to the host, and ends the CTA's others."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2109_12626_gb300 import build as B

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def waits(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("waits") / "proj_waits.so")
    r = subprocess.run([B.nvcc(), *B.ARCH, "-O2", "-std=c++17", "-Xcompiler", "-fPIC,-Wall", "-I", B.CSRC, "-shared",
                        os.path.join(ROOT, "tests", "proj_waits.cu"), "-o", so, "-cudart", "static"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return ctypes.CDLL(so)


def test_a_wait_runs_out(waits):
    limit = 20_000_000   # ns
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    answers = torch.full((96,), -1, dtype=torch.int32, device="cuda")
    took = torch.zeros(3, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    rc = waits.run_waits(ctypes.c_uint64(limit), *(ctypes.c_void_p(t.data_ptr()) for t in (err, answers, took)))
    assert rc == 0
    assert answers.tolist() == [0] * 32 + [1] * 32 + [0] * 32
    assert err.item() == 1
    first, ended, settled = took.tolist()
    assert limit < first < 10 * limit       # it waited, and no longer than that
    assert ended < 10 * limit               # not its own limit
    assert 2 * limit <= settled < 20 * limit
    assert torch.ones(1, device="cuda").item() == 1   # the context is as it was
