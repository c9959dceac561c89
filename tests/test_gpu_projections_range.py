"""Activations and slopes at the ends of the operands' range, where a square or
cube of a projection is infinite: the values are the functions' limits."""
import pytest
import torch

import paper_2109_12626_gb300 as dpdr
import proj_util as U
from proj_tiles import tile_size

pytestmark = pytest.mark.gpu

ENDS = [1e4, 1e13, 1e15, 5e19, 1e20, 1e30, 3e38]


@pytest.mark.parametrize("act", list(U.LIPSCHITZ))
@pytest.mark.parametrize("rows,n", [(1, 16), (14, 16), (70, 33), tile_size(152)])
def test_ends_of_the_range(act, rows, n):
    z = torch.tensor([s * v for v in ENDS for s in (1, -1)])
    x = z[torch.arange(rows) % len(z)].reshape(rows, 1).to(torch.bfloat16).cuda()
    w = torch.ones(n, 1, dtype=torch.bfloat16, device="cuda")
    small = torch.full((n, 1), 2.0 ** -40, dtype=torch.bfloat16, device="cuda")
    dy = torch.full((rows, n), 2.0 ** -20, device="cuda")
    new = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    with dpdr.Linear(rows, 1, n, out="float32", grad="float32", act=act) as lin, \
            dpdr.Gated(rows, 1, n, out="float32", grad="float32", act=act) as gat:
        for keep in (False, True):
            y, pre, pre2, h = new(rows, n), new(rows, n), new(rows, 2 * n), new(rows, n)
            db, dx, dg, du = new(n), new(rows, 1), new(n, 1), new(n, 1)
            lin.forward(x, w, y, pre=pre)
            lin.backward(x, w, dy, dx, dbias=db, pre=pre if keep else None)
            gat.forward(x, w, small, h, pre=pre2)
            gat.backward(x, w, small, dy, dw_gate=dg, dw_up=du, pre=pre2 if keep else None)
            lin.sync()
            gat.sync()
            zz = x.double().expand(rows, n)
            value, slope = U.act64(act, zz), U.slope64(act, zz)
            assert torch.allclose(y.double(), value, rtol=1e-5, atol=1e-30)
            # slopes are 0, 1 or, of no activation, 1
            assert torch.allclose(dx.double(), (dy.double() * slope).sum(1, keepdim=True), rtol=2.0 ** -7, atol=1e-30)
            assert torch.allclose(db.double(), (dy.double() * slope).sum(0), rtol=1e-5, atol=1e-30)
            # h overflows where z z 2^-40 does; nothing is NaN
            assert not torch.isnan(h).any()
