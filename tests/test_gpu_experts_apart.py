"""Experts on the GPU: tokens of a call, and calls of a plan, do not reach into each
other, whatever infinities and NaN they hold."""
import pytest
import torch

import proj_util as U
from test_gpu_experts import layer64, make, pkg, run  # noqa: F401

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("weights,dtype", [("int8", "bfloat16"), ("int8", "float16"), (None, "float16")])
@pytest.mark.parametrize("d", [64, 192, 2880, 100])
def test_rows_of_8_bit_weights_stay_apart(pkg, d, weights, dtype):  # noqa: F811
    """A token's values that are no numbers change no other token's result: the last
    piece of its row of weights (n_model modulo 128 between 1 and 64, mostly) takes
    nothing from the row behind, of this call or of an earlier, longer one."""
    x, router, w, scale = make(40, d, 96, 8, 8, dtype, weights, d + 1)
    with pkg.Experts(40, d, 96, 8, 2, dtype, out="float32", weights=weights or dtype) as plan:
        for rows in (1, 2, 8, 9, 39, 40):
            first, chosen, _ = run(pkg, x[:rows], router, w, scale, 2, out="float32", plan=plan)
            want, _, _, bound, _ = layer64(x[:rows], router, w, scale, 2, 0, "silu", True, chosen)
            U.close("y", first, want, bound, "float32")
            for bad in BAD:
                longer = torch.full_like(x, bad)
                run(pkg, longer, router, w, scale, 2, out="float32", plan=plan)
                again = run(pkg, x[:rows], router, w, scale, 2, out="float32", plan=plan)[0]
                assert torch.equal(again, first), "an earlier call's rows show"
                if rows == 1:
                    continue
                for at in (0, rows // 2, rows - 1):
                    v = x[:rows].clone()
                    v[at] = bad
                    y = run(pkg, v, router, w, scale, 2, out="float32", plan=plan)[0]
                    keep = torch.arange(rows, device="cuda") != at
                    # where long sums are cut depends on what all tokens chose: by the bound
                    U.close("y", y[keep], want[keep], bound[keep], "float32")
                    assert not bool(torch.isfinite(y[at]).any())
