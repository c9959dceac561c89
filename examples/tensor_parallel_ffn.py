"""A gated feed-forward block split over p virtual ranks of one GPU, forward and
backward: what each rank computes, and the reductions between them.

Rank r holds the rows [r H, (r + 1) H) of w_gate and w_up and the same columns
of w_down (H = hidden / p).  Forward, every rank computes its H hidden features
from the same x (``Gated``), then its float32 share of the output (``Linear``,
whose sum over the ranks is the output); ``Plan.allreduce`` adds the shares up,
in the ranks' tree order, into every rank's copy.  Backward, the gradient of
each rank's hidden features and weights needs that rank's data only, and the
ranks' float32 shares of dx are added up by another all-reduce.

    python examples/tensor_parallel_ffn.py [--ranks 4] [--rows 512] [--model 1024] [--hidden 4096]

checks the result against the block computed as a whole in 64 bits and prints
the time of a pass.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2109_12626_gb300 as dpdr  # noqa: E402


class SplitFeedForward:
    """The block's plans, weights and buffers for up to ``rows`` rows."""

    def __init__(self, ranks, rows, model, hidden, dtype="bfloat16", seed=1):
        if hidden % ranks:
            raise ValueError("hidden is not a multiple of ranks")
        self.ranks, self.rows, self.model, self.share = ranks, rows, model, hidden // ranks
        t = getattr(torch, dtype)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        normal = lambda r, c: torch.empty(r, c, dtype=t, device="cuda").normal_(0, c ** -0.5, generator=g)  # noqa: E731
        self.w_gate, self.w_up = normal(hidden, model), normal(hidden, model)
        self.w_down = normal(model, hidden)
        # plans: types of operands, of results and of gradients
        self.up = dpdr.Gated(rows, model, self.share, dtype, grad="float32", act="silu")
        self.down = dpdr.Linear(rows, self.share, model, dtype, out="float32", grad="float32")
        self.down_in = dpdr.Linear(rows, self.share, model, dtype, out="float32")   # its dx in 16 bits
        self.sum = dpdr.Plan(ranks, rows * model, "float32")
        new = lambda r, c, d: [torch.empty(r, c, dtype=d, device="cuda") for _ in range(ranks)]  # noqa: E731
        f32 = torch.float32
        self.h = new(rows, self.share, t)
        self.kept = new(rows, 2 * self.share, f32)
        self.part, self.y = new(rows, model, f32), new(rows, model, f32)
        self.dh = new(rows, self.share, t)
        self.dx_part, self.dx = new(rows, model, f32), new(rows, model, f32)
        self.dw_gate, self.dw_up = new(self.share, model, f32), new(self.share, model, f32)
        self.dw_down = new(model, self.share, f32)

    def _mine(self, w, r):
        return w[r * self.share:(r + 1) * self.share]

    def forward(self, x):
        """Every rank's copy of the output, float32 [rows, model]."""
        for r in range(self.ranks):
            self.up.forward(x, self._mine(self.w_gate, r), self._mine(self.w_up, r), self.h[r], pre=self.kept[r])
            self.down.forward(self.h[r], self._mine(self.w_down.t(), r).t(), self.part[r])
        self.sum.allreduce(self.part, self.y)
        return self.y

    def backward(self, x, dy):
        """Every rank's copy of dx; the weights' gradients are left in dw_*."""
        for r in range(self.ranks):
            w_down = self._mine(self.w_down.t(), r).t()
            self.down.backward(self.h[r], w_down, dy, dw=self.dw_down[r])
            self.down_in.backward(self.h[r], w_down, dy, dx=self.dh[r])
            self.up.backward(x, self._mine(self.w_gate, r), self._mine(self.w_up, r), self.dh[r],
                             dx=self.dx_part[r], dw_gate=self.dw_gate[r], dw_up=self.dw_up[r], pre=self.kept[r])
        self.sum.allreduce(self.dx_part, self.dx)
        return self.dx

    def sync(self):
        for plan in (self.up, self.down, self.down_in, self.sum):
            plan.sync()

    def close(self):
        for plan in (self.up, self.down, self.down_in, self.sum):
            plan.close()


def whole(block, x, dy):
    """The block as a whole in 64 bits: y, dx and the weights' gradients."""
    x, wg, wu, wd = (v.double().requires_grad_(True) for v in (x, block.w_gate, block.w_up, block.w_down))
    y = (torch.nn.functional.silu(x @ wg.t()) * (x @ wu.t())) @ wd.t()
    return (y.detach(), *torch.autograd.grad((y * dy.double()).sum(), (x, wg, wu, wd)))


def worst(block, x, dy):
    """The largest error of y, dx and the weights' gradients in their norms,
    over all ranks' copies."""
    y, dx, dg, du, dd = whole(block, x, dy)
    off = lambda got, want: ((got.double() - want).norm() / want.norm()).item()  # noqa: E731
    errors = {"y": max(off(v, y) for v in block.y), "dx": max(off(v, dx) for v in block.dx)}
    for name, got, want in (("dw_gate", torch.cat(block.dw_gate), dg), ("dw_up", torch.cat(block.dw_up), du),
                            ("dw_down", torch.cat(block.dw_down, 1), dd)):
        errors[name] = off(got, want)
    return errors


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    a = ap.parse_args()
    block = SplitFeedForward(a.ranks, a.rows, a.model, a.hidden)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.empty(a.rows, a.model, device="cuda").normal_(generator=g).to(torch.bfloat16)
    dy = torch.empty(a.rows, a.model, device="cuda").normal_(generator=g)
    for _ in range(3):
        block.forward(x)
        block.backward(x, dy)
    block.sync()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(20):
        block.forward(x)
        block.backward(x, dy)
    end.record()
    block.sync()
    print("%d ranks, %d rows, %d -> %d -> %d: %.1f us forward and backward" % (
        a.ranks, a.rows, a.model, a.hidden, a.model, begin.elapsed_time(end) / 20 * 1e3))
    errors = worst(block, x, dy)
    print("error against 64 bits: " + ", ".join("%s %.2g" % e for e in errors.items()))
    block.close()


if __name__ == "__main__":
    main()
