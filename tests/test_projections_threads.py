"""Calls of the projections' binding from two host threads: each call's
arguments are its own."""
import ctypes
import threading

import pytest
import torch

from paper_2109_12626_gb300 import projections as P


class Tensor:
    """What the binding asks a tensor for."""

    def __init__(self, at, rows, cols, dtype):
        self.at, self.shape, self.dtype = at, torch.Size((rows, cols)), dtype

    def dim(self):
        return 2

    def get_device(self):
        return 0

    def data_ptr(self):
        return self.at

    def stride(self):
        return (self.shape[1], 1)


class Library:
    """Calls that wait for each other before they read their records."""

    def __init__(self, threads):
        self.together = threading.Barrier(threads)
        self.seen = {}

    def dpdr_linear_plan(self, *a):
        return 1

    dpdr_gated_plan = dpdr_linear_plan

    def dpdr_proj_destroy(self, h):
        pass

    def record(self, at):
        return tuple(ctypes.cast(at, ctypes.POINTER(ctypes.c_int64))[i] for i in range(3)) if at else None

    def call(self, h, rows, *args):
        self.together.wait(20)
        found = [self.record(a) for a in args if a and a > 1 << 20]
        self.together.wait(20)
        self.seen[threading.get_ident()] = found
        return 0

    dpdr_linear = dpdr_gated = dpdr_linear_backward = dpdr_gated_backward = call


@pytest.mark.parametrize("what", ["linear", "gated", "linear backward", "gated backward"])
def test_two_threads(monkeypatch, what):
    L = Library(2)
    monkeypatch.setattr(P, "lib", lambda: L)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    plan = (P.Linear if "linear" in what else P.Gated)(8, 16, 24)
    b, want, errors = torch.bfloat16, {}, []

    def run(i):
        try:
            rows = 3 + i
            t = lambda n, r, c: Tensor((i * 100 + n + 1) << 8, r, c, b)  # noqa: E731
            x, w, w2, y = t(1, rows, 16), t(2, 24, 16), t(3, 24, 16), t(4, rows, 24)
            given = [x, w, y] if "linear" in what else [x, w, w2, y]
            want[threading.get_ident()] = [(v.at, v.shape[1], 1) for v in given]
            (plan.backward if "backward" in what else plan.forward)(*given, stream=7)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    plan.close()
    assert not errors and len(L.seen) == 2
    assert L.seen == want
