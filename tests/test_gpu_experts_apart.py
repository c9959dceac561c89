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


@pytest.mark.parametrize("weights,dtype,out", [(None, "bfloat16", None), (None, "bfloat16", "float32"), (None, "float16", "float32"),
                                               ("int8", "bfloat16", None), ("int8", "float16", "float32")])
@pytest.mark.parametrize("rows", [2, 5, 8, 9, 40])
@pytest.mark.parametrize("pitch", [0, 1])
def test_an_expert_reaches_those_that_chose_it(pkg, rows, pitch, weights, dtype, out):  # noqa: F811
    """Infinities and NaN among an expert's weights and scales stay out of the results of
    tokens that did not choose it, and of the features whose rows have none."""
    d, h, total = 192, 72, 8
    x, router, w, scale = make(rows, d, h, total, total, dtype, weights, rows + 50, pitch)
    _, chosen, _ = run(pkg, x, router, w, scale, 2, out=out, weights=weights)
    some = [e for e in range(total) if 0 < int((chosen == e).any(dim=1).sum()) < rows][0]
    took = (chosen == some).any(dim=1)
    want, _, _, bound, _ = layer64(x, router, w, scale, 2, 0, "silu", True, chosen)
    kind = out or dtype
    for bad in BAD:
        for where in ("down", "down scale", "gate"):
            v, s = [t.clone() for t in w], list(scale)   # rows without a pitch
            if pitch:
                v = [a.new_empty(total, a.shape[1], a.shape[2] + pitch)[:, :, :a.shape[2]].copy_(a) for a in w]
            if where == "down scale":
                if weights is None:
                    continue
                s[2] = s[2].clone()
                s[2][some, 3] = bad
            elif where == "down":
                if weights == "int8":
                    continue
                v[2][some, 3, 5] = bad
            elif weights == "int8":
                s[0] = s[0].clone()
                s[0][some, 7] = float("nan")
            else:
                v[0][some, 7, 11] = float("nan")
            y, c, _ = run(pkg, x, router, v, s, 2, out=out, weights=weights)
            assert torch.equal(c, chosen)
            U.close("y", y[~took], want[~took], bound[~took], kind)
            if where == "gate":
                assert not bool(torch.isfinite(y[took]).any())
                continue
            keep = torch.arange(d, device="cuda") != 3
            assert not bool(torch.isfinite(y[took][:, 3]).any())
            U.close("y", y[took][:, keep], want[took][:, keep], bound[took][:, keep], kind)
