"""Experts on the GPU: how many bits of the hidden values enter the last product."""
import pytest
import torch

import proj_util as U
from test_gpu_experts import pkg, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,weights,out", [("bfloat16", None, "bfloat16"), ("bfloat16", None, "float32"),
                                               ("bfloat16", "int8", "bfloat16"), ("bfloat16", "int8", "float32"),
                                               ("float16", "int8", "float16"), ("float16", "int8", "float32"),
                                               ("float16", None, "float16"), ("float16", None, "float32")])
@pytest.mark.parametrize("rows", [1, 3, 8, 9, 17, 33, 64])
@pytest.mark.parametrize("d,h,pitch", [(3, 2, 0), (200, 136, 0), (131, 67, 1)])
def test_what_is_left_where_products_cancel(pkg, rows, d, h, pitch, dtype, weights, out):  # noqa: F811
    """Two hidden values of 23 bits whose difference is the last of these:

        (1 + 2^-12) (1 + 2^-10) - (1 + 2^-10 + 2^-12) 1 = 2^-22

    Every product and sum on the way has at most 23 bits, so none rounds; the tensor cores
    cut sums off at 2^-23 of their largest product at the most.  Hidden values of 16 bits
    give 0, which is off by 2^-22."""
    a, b = h // 3, h - 1            # where the two lie
    t = U.TYPES[dtype]
    x = torch.zeros(rows, d, device="cuda", dtype=t)
    at = [0, d // 2, d - 1]
    x[:, at[0]], x[:, at[1]], x[:, at[2]] = 1.0, 2.0 ** -10, 2.0 ** -12
    kind = torch.int8 if weights == "int8" else t

    def stack(n, k, ones):
        v = torch.zeros(1, n, k + pitch, device="cuda", dtype=kind)[:, :, :k]
        for i, j, s in ones:
            v[0, i, j] = s
        return v

    gate = stack(h, d, [(a, at[0], 1), (a, at[2], 1), (b, at[0], 1), (b, at[1], 1), (b, at[2], 1)])
    up = stack(h, d, [(a, at[0], 1), (a, at[1], 1), (b, at[0], 1)])
    down = stack(d, h, [(i, a, 1 - 2 * (i % 2)) for i in range(d)] + [(i, b, 2 * (i % 2) - 1) for i in range(d)])
    scale = [torch.ones(1, n, device="cuda") for n in (h, h, d)] if weights else [None] * 3
    y, _, share = run(pkg, x, torch.zeros(1, d, device="cuda", dtype=t), [gate, up, down], scale, 1, act="none", out=out, weights=weights)
    assert bool((share == 1).all())
    want = 2.0 ** -22 * (1.0 - 2.0 * (torch.arange(d, device="cuda") % 2)).expand(rows, -1)
    assert bool(((y.double() - want).abs() < 2.0 ** -23).all()), (float(y.double().abs().min()), float(y.double().abs().max()))
