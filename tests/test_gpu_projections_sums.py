"""Sums of the projections that are long: none of their parts is lost, and
their error does not grow with their length."""
import pytest
import torch

import paper_2109_12626_gb300 as dpdr
import proj_util as U

pytestmark = pytest.mark.gpu


def normal(shape, dtype, seed, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=U.TYPES[dtype], device="cuda").normal_(mean, 1.0, generator=g)


def sums64(pairs, rows, at=1 << 20):
    """sum over the rows of a^T b in 64 bits for each pair of functions of a
    slice of rows, piece by piece"""
    total = [0.0] * len(pairs)
    for r in range(0, rows, at):
        for i, (a, b) in enumerate(pairs):
            total[i] = total[i] + a(slice(r, r + at)).double().t() @ b(slice(r, r + at)).double()
    return total


@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
def test_weight_gradients_over_ten_million_rows(grad):
    """10,000,000 rows, 8 to 16 features: 156,250 steps of 64 rows, whose runs
    number 15,625.  dz is rounded to 16 bits (2^-8 of each term's size at
    most, of random sign), sums and results as everywhere."""
    rows, k, n = 10_000_000, 8, 16
    x, dh = normal((rows, k), "bfloat16", 1), normal((rows, n), "bfloat16", 2)
    pre = normal((rows, 2 * n), "float32", 3)
    wg, wu = normal((n, k), "bfloat16", 4), normal((n, k), "bfloat16", 5)
    dg, du = (torch.empty(n, k, dtype=U.TYPES[grad], device="cuda") for _ in range(2))
    dw, dx = torch.empty_like(dg), torch.empty(rows, k, dtype=U.TYPES[grad], device="cuda")
    with dpdr.Gated(rows, k, n, grad=grad, act="none") as gat, dpdr.Linear(rows, k, n, grad=grad) as lin:
        gat.backward(x, wg, wu, dh, dw_gate=dg, dw_up=du, pre=pre)
        lin.backward(x, wg, dh, dx=dx, dw=dw)
        gat.sync()
        lin.sync()
    want = sums64([(lambda r: dh[r].float() * pre[r, n:], lambda r: x[r]), (lambda r: dh[r].float() * pre[r, :n], lambda r: x[r]),
                   (lambda r: dh[r], lambda r: x[r])], rows)
    for name, got, w in zip(("dw_gate", "dw_up", "dw"), (dg, du, dw), want):
        U.close_in_norm(name, got, w, U.ROUND[grad] + 2 * U.ROUND["bfloat16"] + 2.0 ** -10)
    U.close_in_norm("dx", dx[-1000:], dh[-1000:].double() @ wg.double(), U.ROUND[grad] + 2.0 ** -17)
