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


def positive(rows, cols, dtype, seed, scale=1.0):
    """Values of scale times 0.5 to 1.5: no sum of products cancels."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.rand(rows, cols, generator=g, device="cuda") + 0.5).mul_(scale).to(U.TYPES[dtype])


def check_positive(name, got, want, k, mean, most):
    """Sums of k positive products: the mean of their relative errors, where
    random roundings cancel and a bias does not, and the largest."""
    rel = (got.double() - want) / want
    assert rel.mean().abs().item() <= mean, (name, k, rel.mean().item())
    assert rel.abs().max().item() <= most, (name, k, rel.abs().max().item())


# A run of 640 products, 40 additions that each cut off up to 2^-23 of a sum that
# is half of the run's on average: 2.4e-6 at most; measured 8e-7.  The runs are
# added up rounded, 2^-24 each at most, without a bias.
MEAN32 = 1.5e-6


def most32(k):
    return 4e-6 + (k / 512 + 16) * 2.0 ** -24


@pytest.mark.parametrize("rows,k,n", [(128, 8192, 32768), (16, 8192, 40000), (48, 10000, 20000), (100, 65536, 256),
                                      (300, 20000, 264), (1, 65536, 100), (1300, 8192, 1500), (1300, 641, 1501),
                                      (2100, 20001, 1030)])
def test_float32_results_of_long_sums(rows, k, n):
    """Few rows with one to eight CTAs a sum, and tiles."""
    x, w, w2 = positive(rows, k, "bfloat16", 1), positive(n, k, "bfloat16", 2), positive(n, k, "bfloat16", 3, k ** -1.0)
    y, h = (torch.empty(rows, n, device="cuda") for _ in range(2))
    with dpdr.Linear(rows, k, n, out="float32") as lin, dpdr.Gated(rows, k, n, out="float32", act="relu") as gat:
        lin.forward(x, w, y)
        gat.forward(x, w, w2, h)
        lin.sync()
        gat.sync()
    z = x.double() @ w.double().t()
    check_positive("y", y, z, k, MEAN32, most32(k))
    check_positive("h", h, z * (x.double() @ w2.double().t()), k, 2 * MEAN32, 2 * most32(k) + 2.0 ** -23)


@pytest.mark.parametrize("rows,k,n", [(128, 8192, 32768), (48, 40000, 4000), (100, 65536, 256), (1300, 8192, 1500),
                                      (1300, 40000, 1501)])
def test_float16_loses_no_more_of_longer_sums(rows, k, n):
    """Products of float16 have 22 places, which are cut off near the sum's
    last: 3.4e-6 of a run of 640 is lost (measured over one run; if each of them
    lost half of the sum's last place it would be 2e-5), and half as much again
    is allowed, at every length."""
    x, w = positive(rows, k, "float16", 13, 2.0 ** -4), positive(n, k, "float16", 14, 2.0 ** -4)
    y = torch.empty(rows, n, device="cuda")
    with dpdr.Linear(rows, k, n, "float16", out="float32") as lin:
        lin.forward(x, w, y)
        lin.sync()
    check_positive("y", y, x.double() @ w.double().t(), k, 5e-6, 1e-5 + most32(k))


@pytest.mark.parametrize("rows,k,n", [(65536, 256, 256), (1 << 20, 64, 130), (300000, 264, 24), (9000, 2000, 2000)])
def test_float32_weight_gradients_of_long_sums(rows, k, n):
    """dz is dy for the linear operator; for the gated one with w_up's
    projection kept as 1 and no activation dg is dh, and du, of a gate kept as
    2, 2 dh: no rounding of theirs."""
    x, dy, w = positive(rows, k, "bfloat16", 4), positive(rows, n, "bfloat16", 5), positive(n, k, "bfloat16", 6)
    pre = torch.cat([torch.full((rows, n), 2.0, device="cuda"), torch.ones(rows, n, device="cuda")], 1)
    dw, dg, du = (torch.empty(n, k, device="cuda") for _ in range(3))
    with dpdr.Linear(rows, k, n, grad="float32") as lin, dpdr.Gated(rows, k, n, grad="float32", act="none") as gat:
        lin.backward(x, w, dy, dw=dw)
        gat.backward(x, w, w, dy, dw_gate=dg, dw_up=du, pre=pre)
        lin.sync()
        gat.sync()
    want = sums64([(lambda r: dy[r], lambda r: x[r])], rows)[0]
    for name, got, f in (("dw", dw, 1), ("dw_gate", dg, 1), ("dw_up", du, 2)):
        check_positive(name, got, f * want, rows, MEAN32, most32(rows))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_16_bit_weight_gradients_over_millions_of_rows(dtype):
    """Runs of 16,384 products cut off 4e-5 of a sum; the results' roundings
    (2^-9, 2^-12 of them and less) have no bias over the 6,240 elements, which
    columns of different sizes spread over more than an octave."""
    rows, k, n = 3_000_000, 48, 130
    g = torch.Generator(device="cuda").manual_seed(12)
    spread = lambda c: 0.7 + 0.8 * torch.rand(c, generator=g, device="cuda")  # noqa: E731
    x = positive(rows, k, "float32", 7, 2.0 ** -4).mul_(spread(k)).to(U.TYPES[dtype])
    dy = positive(rows, n, "float32", 8, 2.0 ** -4).mul_(spread(n)).to(U.TYPES[dtype])
    w = positive(n, k, dtype, 9)
    pre = torch.ones(rows, 2 * n, device="cuda")
    dw, dg, du = (torch.empty(n, k, dtype=U.TYPES[dtype], device="cuda") for _ in range(3))
    with dpdr.Linear(rows, k, n, dtype) as lin, dpdr.Gated(rows, k, n, dtype, act="none") as gat:
        lin.backward(x, w, dy, dw=dw)
        gat.backward(x, w, w, dy, dw_gate=dg, dw_up=du, pre=pre)
        lin.sync()
        gat.sync()
    want = sums64([(lambda r: dy[r], lambda r: x[r])], rows)[0]
    for name, got in (("dw", dw), ("dw_gate", dg), ("dw_up", du)):
        check_positive(name, got, want, rows, 5e-5 + U.ROUND[dtype] / 16, 1e-4 + U.ROUND[dtype])


@pytest.mark.parametrize("rows,n", [(1300, 1500), (1300, 1501), (100, 300), (20, 77)])
def test_16_bit_sums_of_several_runs(rows, n):
    """Rows of more elements than a run of 16-bit results holds, everything
    that a finished sum may need, both operators, forward and backward."""
    import test_gpu_projections as T
    k = 33_000 if rows > 128 else 300_000
    T.linear_case(rows, k, n, act="silu", pre=True)
    T.gated_case(rows, k, n // 2, "float16", act="gelu")
    T.linear_gradient_case(rows, k, n, act="gelu_tanh")
    T.gated_gradient_case(rows, k, n // 2)


def test_long_sums_repeat_themselves():
    """The same bits twice, of runs in turn and of tiles."""
    for rows, k, n in ((128, 8192, 9000), (100, 65536, 256), (1300, 2000, 1500)):
        x, w = normal((rows, k), "bfloat16", 10), normal((n, k), "bfloat16", 11)
        a, b = (torch.empty(rows, n, device="cuda") for _ in range(2))
        with dpdr.Linear(rows, k, n, out="float32") as lin:
            lin.forward(x, w, a)
            lin.forward(x, w, b)
            lin.sync()
        assert torch.equal(a, b)
