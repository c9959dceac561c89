"""What answers tokens next to a split model's reductions with fewer bytes:
``quantise`` (rows rounded to 8-bit integers), ``Linear8`` (their product with
8-bit weights) and ``Experts`` (a layer of experts for a few tokens).  A thin
binding of ``dpdr_quantise``, ``dpdr_integer_*`` and ``dpdr_experts*`` of
``include/dpdr.h``: torch supplies device memory and streams, and the caller
owns every buffer.

    dpdr.quantise(sums, q, scale)                          # what a reduction left
    with dpdr.Linear8(rows, n_in, n_out, out="float32") as proj:
        proj.forward(q, scale, w, w_scale, partial)        # one rank's share
    with dpdr.Experts(rows, n_model, n_hidden, 64, 8, first=16, local=16, out="float32") as moe:
        moe.forward(x, router, w_gate, w_up, w_down, partial)
"""
from __future__ import annotations

import ctypes

from ._native import DPDR_INT8, DpdrError, _check, _stream, lib
from .projections import ACTIVATIONS, OPERANDS, RESULTS, _Projection


def _known(what, name, known):
    if name not in known:
        raise ValueError("%s: %r is none of %s" % (what, name, ", ".join(known)))


def quantise(x, q, scale, stream=None) -> None:
    """q, scale <- x's rows rounded to 8-bit integers: scale = a / 127 with a
    the largest size in the row, q = 127 x / a rounded, halves to even.  x
    [rows, n] in bfloat16, float16 or float32, any strides; q int8 [rows, n];
    scale float32 [rows].  Weights are rounded alike, a row a channel."""
    if _codes is None:
        _first()
    code = _codes.get(x.dtype)
    if code is None:
        raise TypeError("x is %s, not one of %s" % (x.dtype, ", ".join(RESULTS)))
    if x.dim() != 2:
        raise ValueError("x has %d dimensions, not 2" % x.dim())
    rows, n = x.shape
    if q.dtype is not _int8 or scale.dtype is not _float32:
        raise TypeError("q is %s and scale %s, not int8 and float32" % (q.dtype, scale.dtype))
    if q.shape != x.shape or scale.shape != (rows,):
        raise ValueError("q is %s and scale %s for an x of %s" % (tuple(q.shape), tuple(scale.shape), tuple(x.shape)))
    at = x.get_device()
    if at < 0 or at != q.get_device() or at != scale.get_device() or at != _device():
        raise ValueError("x, q and scale are not all on the current device")
    if rows > 1 and scale.stride(0) != 1:
        raise ValueError("scale: contiguous elements are needed")
    r = _records(x.data_ptr(), *x.stride(), q.data_ptr(), *q.stride())
    base = ctypes.addressof(r)
    rc = _quantise(rows, n, code, base, base + 24, scale.data_ptr(), _stream(stream))
    if rc:
        _check(rc, "dpdr_quantise")


_records = ctypes.c_int64 * 6   # x and q as dpdr_matrix records
_codes = _int8 = _float32 = _device = _quantise = None


def _first():
    """What a call looks up once."""
    global _codes, _int8, _float32, _device, _quantise
    import torch
    _quantise = lib().dpdr_quantise
    _int8, _float32 = torch.int8, torch.float32
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _codes = {getattr(torch, name): code for name, code in RESULTS.items()}


class _Serving(_Projection):
    """A plan with its own calls to wait for it and to free it."""

    _end = ()

    def _start(self, make, *args):
        import torch
        L = lib()
        h = getattr(L, make)(*args)
        if not h:
            raise DpdrError(L.dpdr_last_error(), make)
        self._h = h
        self._device = torch.cuda.current_device()
        self._int8, self._float32, self._int32 = torch.int8, torch.float32, torch.int32
        self._local = _local()

    def close(self) -> None:
        if getattr(self, "_h", None):
            getattr(lib(), self._end[1])(self._h)
            self._h = None

    def sync(self, stream=None) -> None:
        """Wait for the stream; raise DpdrError if a kernel failed."""
        _check(getattr(lib(), self._end[0])(self._h, _stream(stream)), self._end[0])


def _local():
    import threading
    return threading.local()


class Linear8(_Serving):
    """y = (x w^T) x_scale w_scale + bias + residual: x int8 [rows, n_in], w
    int8 [n_out, n_in], x_scale [rows], w_scale and bias [n_out] in float32.

    ``out`` is the type of y and the residual ("bfloat16", "float16",
    "float32").  Sums are exact.  x, w and the residual may have any strides.
    x_scale w_scale has to be a normal float32 number or 0."""

    _end = ("dpdr_integer_sync", "dpdr_integer_destroy")
    _args = 4

    def __init__(self, max_rows: int, n_in: int, n_out: int, out="bfloat16"):
        import torch
        _known("out", out, RESULTS)
        self._start("dpdr_integer_plan", int(max_rows), int(n_in), int(n_out), RESULTS[out])
        self._forward = lib().dpdr_integer_linear
        self.max_rows, self.n_in, self.n_out, self.out = int(max_rows), int(n_in), int(n_out), out
        self._result = getattr(torch, out)

    def forward(self, x, x_scale, w, w_scale, y, bias=None, residual=None, stream=None) -> None:
        """y <- (x w^T) x_scale w_scale + bias + residual (y may be the
        residual itself)."""
        rows, k, n = self._rows(x), self.n_in, self.n_out
        r = self._records()
        rc = self._forward(self._h, rows, self._matrix(r, 0, "x", x, rows, k, self._int8),
                           self._vector("x_scale", x_scale, rows, self._float32),
                           self._matrix(r, 1, "w", w, n, k, self._int8),
                           self._vector("w_scale", w_scale, n, self._float32),
                           self._vector("bias", bias, n, self._float32),
                           self._matrix(r, 2, "residual", residual, rows, n, self._result),
                           self._matrix(r, 3, "y", y, rows, n, self._result), _stream(stream))
        if rc:
            _check(rc, "dpdr_integer_linear")


class Experts(_Serving):
    """y = sum over a token's chosen experts e that are here of
    share_e (act(x w_gate[e]^T) * (x w_up[e]^T)) w_down[e]^T.

    ``experts`` in all, ``top`` chosen for each token by the scores x router^T
    (equal ones: the lower number), with shares exp(score) over the sum of
    these, of the chosen (``normalise``) or of all.  The plan's rank holds the
    ``local`` experts from ``first`` on.  ``dtype`` is the type of x and the
    router, ``weights`` of the experts (the same, or "int8" with a scale for
    each of their rows), ``out`` of y (the same, or "float32").  At most 64
    rows."""

    _end = ("dpdr_experts_sync", "dpdr_experts_destroy")
    _args = 3

    def __init__(self, max_rows: int, n_model: int, n_hidden: int, experts: int, top: int, dtype="bfloat16",
                 out=None, weights=None, act="silu", first: int = 0, local=None, normalise: bool = True):
        import torch
        out, weights = out or dtype, weights or dtype
        held = dict(OPERANDS, int8=DPDR_INT8)
        for what, name, known in (("dtype", dtype, OPERANDS), ("out", out, RESULTS), ("weights", weights, held),
                                  ("act", act, ACTIVATIONS)):
            _known(what, name, known)
        local = int(experts) - int(first) if local is None else int(local)
        self._start("dpdr_experts_plan", int(max_rows), int(n_model), int(n_hidden), int(experts), int(top),
                    int(first), local, OPERANDS[dtype], held[weights], RESULTS[out], ACTIVATIONS[act],
                    int(bool(normalise)))
        self._forward = lib().dpdr_experts
        self.max_rows, self.n_model, self.n_hidden = int(max_rows), int(n_model), int(n_hidden)
        self.experts, self.top, self.first, self.local = int(experts), int(top), int(first), local
        self.dtype, self.out, self.weights, self.act, self.normalise = dtype, out, weights, act, bool(normalise)
        self._operand, self._result, self._held = (getattr(torch, t) for t in (dtype, out, weights))

    def _stack(self, records, i, name, t, rows, cols):
        """Weights number i as a dpdr_matrices record; its address."""
        if t.dtype is not self._held or t.shape != (self.local, rows, cols) or t.get_device() != self._device:
            self._unfit(name, t, (self.local, rows, cols), self._held)
        r, at = records
        base = 3 * self._args + 4 * i
        r[base] = t.data_ptr()
        r[base + 1], r[base + 2], r[base + 3] = t.stride()
        return at[0] + 8 * base

    def _records(self):
        try:
            return self._local.records
        except AttributeError:
            r = (ctypes.c_int64 * (3 * self._args + 12))()
            base = ctypes.addressof(r)
            self._local.records = r, [base + 24 * i for i in range(self._args)]
            return self._local.records

    def _pairs(self, name, t, rows, dtype):
        """chosen or share: contiguous, rows by top."""
        if t is None:
            return 0
        if t.dtype is not dtype or t.shape != (rows, self.top) or t.get_device() != self._device:
            self._unfit(name, t, (rows, self.top), dtype)
        if not t.is_contiguous():
            raise ValueError("%s: the plan wants contiguous elements" % name)
        return t.data_ptr()

    def _scale(self, name, t, channels):
        if t is None:
            return 0
        if t.dtype is not self._float32 or t.shape != (self.local, channels) or t.get_device() != self._device:
            self._unfit(name, t, (self.local, channels), self._float32)
        if not t.is_contiguous():
            raise ValueError("%s: the plan wants contiguous elements" % name)
        return t.data_ptr()

    def forward(self, x, router, w_gate, w_up, w_down, y, gate_scale=None, up_scale=None, down_scale=None,
                chosen=None, share=None, stream=None) -> None:
        """y <- the layer's result for x [rows, n_model]; router [experts,
        n_model], w_gate and w_up [local, n_hidden, n_model], w_down [local,
        n_model, n_hidden], the scales of 8-bit weights [local, their rows] in
        float32.  chosen (int32) and share (float32), [rows, top]: which experts
        each token takes and with what share, largest first."""
        rows, d, h = self._rows(x), self.n_model, self.n_hidden
        r = self._records()
        rc = self._forward(self._h, rows, self._matrix(r, 0, "x", x, rows, d, self._operand),
                           self._matrix(r, 1, "router", router, self.experts, d, self._operand),
                           self._stack(r, 0, "w_gate", w_gate, h, d), self._stack(r, 1, "w_up", w_up, h, d),
                           self._stack(r, 2, "w_down", w_down, d, h),
                           self._scale("gate_scale", gate_scale, h), self._scale("up_scale", up_scale, h),
                           self._scale("down_scale", down_scale, d),
                           self._matrix(r, 2, "y", y, rows, d, self._result),
                           self._pairs("chosen", chosen, rows, self._int32),
                           self._pairs("share", share, rows, self._float32), _stream(stream))
        if rc:
            _check(rc, "dpdr_experts")
