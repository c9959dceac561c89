"""A block that answers tokens, split over p virtual ranks: a projection held in
8-bit integers, row-parallel, and a layer of experts, expert-parallel.  Both leave
float32 partials on every rank that a reduction-to-all adds up:

    q, s     = quantise(x's columns of this rank)            8-bit integers, a scale a token
    partial  = (q w_r^T) s w_scale_r                         Linear8, float32
    y        = reduction of the partials, to bfloat16
    partial' = sum of this rank's chosen experts of y        Experts, float32
    z        = reduction of the partials'

    python examples/expert_parallel_tokens.py [ranks tokens n_model n_hidden experts top]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2109_12626_gb300 as dpdr  # noqa: E402


class SplitTokens:
    """Weights, plans and buffers of all ranks.  n_model is a multiple of the ranks,
    and so are the experts."""

    def __init__(self, ranks, tokens, n_model, n_hidden, experts, top, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        new = lambda dt, *s: torch.empty(*s, device="cuda", dtype=dt)  # noqa: E731
        self.ranks, self.tokens, self.cut, self.held = ranks, tokens, n_model // ranks, experts // ranks
        self.w, self.w_scale = [], []
        for r in range(ranks):   # a rank's columns of the weights, rounded row by row
            q, s = new(torch.int8, n_model, self.cut), new(torch.float32, n_model)
            dpdr.quantise(normal(n_model, self.cut) * n_model ** -0.5, q, s)
            self.w.append(q)
            self.w_scale.append(s)
        self.router = (normal(experts, n_model) * n_model ** -0.5).bfloat16()
        self.experts = [[(normal(self.held, n_hidden, n_model) * n_model ** -0.5).bfloat16(),
                         (normal(self.held, n_hidden, n_model) * n_model ** -0.5).bfloat16(),
                         (normal(self.held, n_model, n_hidden) * n_hidden ** -0.5).bfloat16()] for _ in range(ranks)]
        self.proj = dpdr.Linear8(tokens, self.cut, n_model, out="float32")
        self.layers = [dpdr.Experts(tokens, n_model, n_hidden, experts, top, "bfloat16", out="float32",
                                    first=r * self.held, local=self.held) for r in range(ranks)]
        self.plan = dpdr.Plan(ranks, tokens * n_model, "float32")
        self.q = [new(torch.int8, tokens, self.cut) for _ in range(ranks)]
        self.s = [new(torch.float32, tokens) for _ in range(ranks)]
        self.partial, self.y, self.z = ([new(torch.float32, tokens, n_model) for _ in range(ranks)] for _ in range(3))
        self.h = new(torch.bfloat16, tokens, n_model)

    def forward(self, x):
        """z on every rank, for x [tokens, n_model] whose columns the ranks share."""
        for r in range(self.ranks):
            dpdr.quantise(x[:, r * self.cut:(r + 1) * self.cut], self.q[r], self.s[r])
            self.proj.forward(self.q[r], self.s[r], self.w[r], self.w_scale[r], self.partial[r])
        self.plan.allreduce([t.view(-1) for t in self.partial], [t.view(-1) for t in self.y])
        self.h.copy_(self.y[0])
        for r in range(self.ranks):
            self.layers[r].forward(self.h, self.router, *self.experts[r], self.partial[r])
        self.plan.allreduce([t.view(-1) for t in self.partial], [t.view(-1) for t in self.z])
        return self.z

    def sync(self):
        self.proj.sync()
        for layer in self.layers:
            layer.sync()
        self.plan.sync()

    def close(self):
        for p in (self.proj, self.plan, *self.layers):
            p.close()


def worst(block, x):
    """The largest errors of y and z, of their norms, against the same block in 64
    bits (of z, from the rounded y that the experts get)."""
    y = sum(q.double() @ w.double().t() * s.double()[:, None] * ws.double()
            for q, w, s, ws in zip(block.q, block.w, block.s, block.w_scale))
    h = block.h.double()
    scores = h @ block.router.double().t()
    top = block.layers[0].top
    picked, order = scores.sort(dim=1, descending=True, stable=True)
    share = torch.softmax(picked[:, :top], dim=1)
    z = torch.zeros_like(h)
    for t in range(block.tokens):
        for s, e in zip(share[t], order[t, :top].tolist()):
            gate, up, down = (w[e % block.held].double() for w in block.experts[e // block.held])
            z[t] += s * (down @ (torch.nn.functional.silu(gate @ h[t]) * (up @ h[t])))
    error = lambda got, want: float((got.double() - want).norm() / want.norm())  # noqa: E731
    return {"y": max(error(t, y) for t in block.y), "z": max(error(t, z) for t in block.z)}


def main():
    sizes = [int(a) for a in sys.argv[1:]] or [4, 8, 512, 256, 16, 2]
    block = SplitTokens(*sizes)
    x = torch.randn(sizes[1], sizes[2], device="cuda")
    block.forward(x)
    block.sync()
    print("ranks %d: errors against 64 bits %s" % (sizes[0], worst(block, x)))
    block.close()


if __name__ == "__main__":
    main()
