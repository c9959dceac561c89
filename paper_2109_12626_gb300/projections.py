"""Projections of a split model next to its reductions: ``Linear`` (matrix
product with bias, activation and residual) and ``Gated`` (two projections,
the activation and their product), each with its gradients.  A thin binding
of ``dpdr_linear*`` and ``dpdr_gated*`` of ``include/dpdr.h``: torch supplies
device memory and streams, and the caller owns every buffer.

    with dpdr.Linear(rows, n_in, n_out, "bfloat16", out="float32") as proj:
        proj.forward(x, w, partial)      # one rank's share, float32
    plan.allreduce(partials, sums)       # a Plan adds the ranks' shares up
"""
from __future__ import annotations

import ctypes
import threading

from ._native import (DPDR_BFLOAT16, DPDR_FLOAT16, DPDR_FLOAT32, DpdrError, _check, _stream, lib)

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4, "sigmoid": 5}
OPERANDS = {"bfloat16": DPDR_BFLOAT16, "float16": DPDR_FLOAT16}
RESULTS = dict(OPERANDS, float32=DPDR_FLOAT32)


class _Projection:
    """What both operators share: the plan handle, and matrix arguments."""

    _plan = ""
    _calls = ()
    _args = 0

    def __init__(self, max_rows: int, n_in: int, n_out: int, dtype="bfloat16", out=None,
                 grad=None, act="none"):
        import torch
        out, grad = out or dtype, grad or dtype
        for what, name, known in (("dtype", dtype, OPERANDS), ("out", out, RESULTS),
                                  ("grad", grad, RESULTS), ("act", act, ACTIVATIONS)):
            if name not in known:
                raise ValueError("%s: %r is none of %s" % (what, name, ", ".join(known)))
        L = lib()
        h = getattr(L, self._plan)(int(max_rows), int(n_in), int(n_out), OPERANDS[dtype],
                                   RESULTS[out], RESULTS[grad], ACTIVATIONS[act])
        if not h:
            raise DpdrError(L.dpdr_last_error(), self._plan)
        self._h = h
        self._forward, self._backward = (getattr(L, f) for f in self._calls)
        self._device = torch.cuda.current_device()
        self.max_rows, self.n_in, self.n_out = int(max_rows), int(n_in), int(n_out)
        self.dtype, self.out, self.grad, self.act = dtype, out, grad, act
        self._operand, self._result, self._gradient = (getattr(torch, t) for t in (dtype, out, grad))
        self._float32 = torch.float32
        self._local = threading.local()

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().dpdr_proj_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def sync(self, stream=None) -> None:
        """Wait for the stream; raise DpdrError if a kernel's bounded wait expired."""
        _check(lib().dpdr_proj_sync(self._h, _stream(stream)), "dpdr_proj_sync")

    def _records(self):
        """dpdr_matrix records (address, row stride, column stride) of a call's
        arguments, filled in anew by each call, and their addresses: this
        thread's, since a call lets other threads run while it reads them."""
        try:
            return self._local.records
        except AttributeError:
            r = (ctypes.c_int64 * (3 * self._args))()
            base = ctypes.addressof(r)
            self._local.records = r, [base + 24 * i for i in range(self._args)]
            return self._local.records

    def _matrix(self, records, i, name, t, rows, cols, dtype):
        """Argument number i as a record; its address, 0 for None."""
        if t is None:
            return 0
        if t.dtype is not dtype or t.shape != (rows, cols) or t.get_device() != self._device:
            self._unfit(name, t, (rows, cols), dtype)
        r, at = records
        r[3 * i] = t.data_ptr()
        r[3 * i + 1], r[3 * i + 2] = t.stride()
        return at[i]

    def _vector(self, name, t, n, dtype):
        if t is None:
            return 0
        if t.dtype is not dtype or t.shape != (n,) or t.get_device() != self._device:
            self._unfit(name, t, (n,), dtype)
        if n > 1 and t.stride(0) != 1:
            raise ValueError("%s: the plan wants contiguous elements" % name)
        return t.data_ptr()

    def _unfit(self, name, t, shape, dtype):
        if t.dtype is not dtype:
            raise TypeError("%s is %s, the plan wants %s" % (name, t.dtype, dtype))
        if t.shape != shape:
            raise ValueError("%s is %s, the plan wants %s" % (name, tuple(t.shape), shape))
        raise ValueError("%s is not on the plan's device" % name)

    def _rows(self, x):
        if x.dim() != 2:
            raise ValueError("x has %d dimensions, not 2" % x.dim())
        return x.shape[0]


class Linear(_Projection):
    """y = act(x w^T + bias) + residual: x [rows, n_in], w [n_out, n_in].

    ``dtype`` is the operands' type ("bfloat16", "float16"), ``out`` that of
    y, the residual and dy, ``grad`` that of the gradients: the operands' or
    "float32".  ``act``: "none", "relu", "gelu", "gelu_tanh", "silu" or
    "sigmoid".  Any number of rows up to ``max_rows`` goes through a plan."""

    _plan = "dpdr_linear_plan"
    _calls = ("dpdr_linear", "dpdr_linear_backward")
    _args = 7

    def forward(self, x, w, y, bias=None, residual=None, pre=None, stream=None) -> None:
        """Writes y; y may be the residual.  ``pre`` (float32 [rows, n_out])
        keeps x w^T + bias for the backward call."""
        rows, k, n = self._rows(x), self.n_in, self.n_out
        m, q = self._matrix, self._records()
        rc = self._forward(self._h, rows, m(q, 0, "x", x, rows, k, self._operand),
                           m(q, 1, "w", w, n, k, self._operand),
                           self._vector("bias", bias, n, self._operand),
                           m(q, 2, "residual", residual, rows, n, self._result),
                           m(q, 3, "y", y, rows, n, self._result),
                           m(q, 4, "pre", pre, rows, n, self._float32), _stream(stream))
        if rc:
            raise DpdrError(rc, "dpdr_linear")

    def backward(self, x, w, dy, dx=None, dw=None, dbias=None, bias=None, pre=None,
                 stream=None) -> None:
        """Writes those of dx, dw and dbias that are given.  Without ``pre``
        the projection is computed again, for which it needs the bias."""
        rows, k, n = self._rows(x), self.n_in, self.n_out
        m, q = self._matrix, self._records()
        rc = self._backward(self._h, rows, m(q, 0, "x", x, rows, k, self._operand),
                            m(q, 1, "w", w, n, k, self._operand),
                            self._vector("bias", bias, n, self._operand),
                            m(q, 2, "dy", dy, rows, n, self._result),
                            m(q, 3, "pre", pre, rows, n, self._float32),
                            m(q, 4, "dx", dx, rows, k, self._gradient),
                            m(q, 5, "dw", dw, n, k, self._gradient),
                            self._vector("dbias", dbias, n, self._gradient),
                            _stream(stream))
        if rc:
            raise DpdrError(rc, "dpdr_linear_backward")


class Gated(_Projection):
    """h = act(x w_gate^T) * (x w_up^T): x [rows, n_in], weights
    [n_hidden, n_in].  Types and activations as for Linear."""

    _plan = "dpdr_gated_plan"
    _calls = ("dpdr_gated", "dpdr_gated_backward")
    _args = 8

    def __init__(self, max_rows, n_in, n_hidden, dtype="bfloat16", out=None, grad=None, act="silu"):
        super().__init__(max_rows, n_in, n_hidden, dtype, out, grad, act)
        self.n_hidden = self.n_out

    def forward(self, x, w_gate, w_up, h, pre=None, stream=None) -> None:
        """Writes h.  ``pre`` (float32 [rows, 2 n_hidden]) keeps both
        projections, the gate's first, for the backward call."""
        rows, k, n = self._rows(x), self.n_in, self.n_out
        m, q = self._matrix, self._records()
        rc = self._forward(self._h, rows, m(q, 0, "x", x, rows, k, self._operand),
                           m(q, 1, "w_gate", w_gate, n, k, self._operand),
                           m(q, 2, "w_up", w_up, n, k, self._operand),
                           m(q, 3, "h", h, rows, n, self._result),
                           m(q, 4, "pre", pre, rows, 2 * n, self._float32), _stream(stream))
        if rc:
            raise DpdrError(rc, "dpdr_gated")

    def backward(self, x, w_gate, w_up, dh, dx=None, dw_gate=None, dw_up=None, pre=None,
                 stream=None) -> None:
        """Writes dx, and dw_gate with dw_up, where given.  Without ``pre``
        the projections are computed again."""
        rows, k, n = self._rows(x), self.n_in, self.n_out
        m, q = self._matrix, self._records()
        rc = self._backward(self._h, rows, m(q, 0, "x", x, rows, k, self._operand),
                            m(q, 1, "w_gate", w_gate, n, k, self._operand),
                            m(q, 2, "w_up", w_up, n, k, self._operand),
                            m(q, 3, "dh", dh, rows, n, self._result),
                            m(q, 4, "pre", pre, rows, 2 * n, self._float32),
                            m(q, 5, "dx", dx, rows, k, self._gradient),
                            m(q, 6, "dw_gate", dw_gate, n, k, self._gradient),
                            m(q, 7, "dw_up", dw_up, n, k, self._gradient), _stream(stream))
        if rc:
            raise DpdrError(rc, "dpdr_gated_backward")
