"""Products of 8-bit integers and rounding to them on the GPU against the
definition: whole numbers exactly, scaled sums to a few roundings."""
import pytest
import torch

import proj_util as U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    from paper_2109_12626_gb300 import build as B
    B.build()
    import paper_2109_12626_gb300 as pkg
    pkg.lib()
    return pkg


def bytes_(g, *shape):
    return torch.randint(-128, 128, shape, device="cuda", generator=g).to(torch.int8)


def lay(v, how):
    """The same values, lying otherwise."""
    if how == "turned":
        return torch.empty(v.shape[1], v.shape[0], device="cuda", dtype=v.dtype).t().copy_(v)
    if how == "slack":
        return torch.full((v.shape[0], v.shape[1] + 16), 99, device="cuda", dtype=v.dtype)[:, :v.shape[1]].copy_(v)
    if how == "odd":
        return torch.full((v.shape[0], v.shape[1] + 5), 99, device="cuda", dtype=v.dtype)[:, 3:v.shape[1] + 3].copy_(v)
    if how == "apart":
        return torch.full((v.shape[0], 2 * v.shape[1]), 99, device="cuda", dtype=v.dtype)[:, ::2].copy_(v)
    return v


def product64(x, w):
    """Whole numbers below 2^53: exact in float64."""
    return x.double() @ w.double().t()


def check(pkg, x, xs, w, ws, out, bias=None, residual=None, plan=None):
    rows, n = x.shape[0], w.shape[0]
    y = torch.full((rows + 2, n + 3), 7.0, device="cuda", dtype=U.TYPES[out])
    own = plan is None
    plan = plan or pkg.Linear8(rows, x.shape[1], n, out=out)
    plan.forward(x, xs, w, ws, y[1:-1, 1:n + 1], bias=bias, residual=residual)
    plan.sync()
    if own:
        plan.close()
    guard = y.clone()
    guard[1:-1, 1:n + 1] = 7.0
    assert bool((guard == 7.0).all()), "written outside the result"
    z = product64(x, w) * xs.double()[:, None] * ws.double()
    want = z + (0 if bias is None else bias.double()) + (0 if residual is None else residual.double())
    # the sum to float32, the scales' product, theirs, two additions: five of 2^-24
    bound = 5 * 2.0 ** -24 * (z.abs() + (0 if bias is None else bias.double().abs()) +
                              (0 if residual is None else residual.double().abs()))
    U.close("y", y[1:-1, 1:n + 1], want, bound, out)
    return y[1:-1, 1:n + 1].clone()


def scales(g, n):
    return torch.rand(n, device="cuda", generator=g) * 0.01 + 0.001


SIZES = [(1, 1, 1), (1, 64, 32), (1, 4096, 1000), (2, 63, 5), (3, 100, 33), (8, 512, 96), (9, 1000, 70), (16, 64, 64),
         (17, 2500, 31), (33, 320, 129), (64, 1024, 257), (64, 65, 40), (65, 64, 32), (100, 1000, 300), (200, 130, 513),
         (257, 2048, 260), (300, 72, 1000), (5, 20000, 48), (70, 20000, 48)]


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("out", ["bfloat16", "float16", "float32"])
def test_against_the_definition(pkg, rows, k, n, out):
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    x, w = bytes_(g, rows, k), bytes_(g, n, k)
    bias = torch.randn(n, device="cuda", generator=g) if (rows + n) % 2 else None
    residual = torch.randn(rows, n, device="cuda", generator=g).to(U.TYPES[out]) if k % 2 == 0 else None
    check(pkg, x, scales(g, rows), w, scales(g, n), out, bias, residual)


@pytest.mark.parametrize("rows", [1, 6, 30, 64, 90, 300])
@pytest.mark.parametrize("how_x,how_w", [("turned", "plain"), ("plain", "turned"), ("slack", "odd"), ("odd", "slack"),
                                         ("apart", "apart"), ("odd", "odd")])
def test_operands_as_they_lie(pkg, rows, how_x, how_w):
    g = torch.Generator(device="cuda").manual_seed(rows)
    for k, n in ((192, 100), (333, 65)):
        x, w = bytes_(g, rows, k), bytes_(g, n, k)
        check(pkg, lay(x, how_x), scales(g, rows), lay(w, how_w), scales(g, n), "float32")


@pytest.mark.parametrize("rows", [1, 2, 3])
@pytest.mark.parametrize("k", [1, 15, 16, 17, 32, 1003, 9000])
def test_tokens_at_any_address(pkg, rows, k):
    """Every place of x and w within 16 bytes, and others' values on both sides."""
    g = torch.Generator(device="cuda").manual_seed(k)
    n = 9
    with pkg.Linear8(rows, k, n, out="float32") as plan:
        for at in range(16):
            x, w = bytes_(g, rows, k + 37)[:, 5 * at % 16:][:, :k], bytes_(g, n, k + 37 - at % 3)[:, at:at + k]
            check(pkg, x, scales(g, rows), w, scales(g, n), "float32", plan=plan)


@pytest.mark.parametrize("rows", [1, 5, 12, 40, 80, 300])
@pytest.mark.parametrize("k", [512, 1024, 4096, 16384, 131071])
def test_sums_are_exact(pkg, rows, k):
    """The largest products there are, sums of one sign and sums that cancel to
    almost nothing."""
    n = 40
    x = torch.full((rows, k), -128, device="cuda", dtype=torch.int8)
    w = torch.full((n, k), -128, device="cuda", dtype=torch.int8)
    w[1::2, k // 2:] = 127
    w[2::4, ::2] = 127
    w[5, :] = 127
    w[6, k // 2:] = 127
    w[6, -1] = 1
    x[1::2, ::3] = 127
    one_x, one_w = torch.ones(rows, device="cuda"), torch.ones(n, device="cuda")
    y = torch.empty(rows, n, device="cuda")
    with pkg.Linear8(rows, k, n, out="float32") as plan:
        plan.forward(x, one_x, w, one_w, y)
        plan.sync()
    # a sum is a whole number that float32 rounds once
    assert torch.equal(y, product64(x, w).float())


def test_results_in_place_on_the_residual(pkg):
    g = torch.Generator(device="cuda").manual_seed(1)
    for rows in (4, 100):
        x, w, xs, ws = bytes_(g, rows, 256), bytes_(g, 96, 256), scales(g, rows), scales(g, 96)
        y = torch.randn(rows, 96, device="cuda", generator=g).to(torch.bfloat16)
        want = check(pkg, x, xs, w, ws, "bfloat16", residual=y.clone())
        with pkg.Linear8(rows, 256, 96) as plan:
            plan.forward(x, xs, w, ws, y, residual=y)
            plan.sync()
        assert torch.equal(y, want)


def test_broadcast_and_turned_residuals(pkg):
    g = torch.Generator(device="cuda").manual_seed(2)
    for rows in (7, 130):
        x, w, xs, ws = bytes_(g, rows, 128), bytes_(g, 72, 128), scales(g, rows), scales(g, 72)
        one = torch.randn(72, device="cuda", generator=g).half()
        check(pkg, x, xs, w, ws, "float16", residual=one.expand(rows, 72))
        check(pkg, x, xs, w, ws, "float16", residual=torch.randn(72, rows, device="cuda", generator=g).half().t())


def test_scales_without_a_value_stay_in_their_place(pkg):
    g = torch.Generator(device="cuda").manual_seed(3)
    for rows in (6, 150):
        x, w, xs, ws = bytes_(g, rows, 96), bytes_(g, 64, 96), scales(g, rows), scales(g, 64)
        plain = check(pkg, x, xs, w, ws, "float32")
        xs[3], ws[10] = float("nan"), float("inf")
        y = torch.empty(rows, 64, device="cuda")
        with pkg.Linear8(rows, 96, 64, out="float32") as plan:
            plan.forward(x, xs, w, ws, y)
            plan.sync()
        assert bool(torch.isnan(y[3]).all()) and not bool(torch.isfinite(y[:, 10]).any())
        y[3], y[:, 10] = plain[3], plain[:, 10]
        assert torch.equal(y, plain)


@pytest.mark.parametrize("rows", [2, 12, 100, 700])
def test_scales_and_bias_at_any_place(pkg, rows):
    """Vectors that start at odd elements of their arrays, and results whose rows do."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x, w = bytes_(g, rows, 320), bytes_(g, 1000, 320)
    xs, ws = scales(g, rows + 1)[1:], scales(g, 1003)[3:]
    bias = torch.randn(1001, device="cuda", generator=g)[1:]
    residual = torch.randn(rows, 1001, device="cuda", generator=g).bfloat16()[:, 1:]
    check(pkg, x, xs, w, ws, "bfloat16", bias, residual)
    check(pkg, x, xs, w, ws, "float32", bias, residual.float())


def test_two_plans_on_two_streams(pkg):
    """Calls of different plans may overlap: each has scratch of its own."""
    g = torch.Generator(device="cuda").manual_seed(10)
    w, ws = bytes_(g, 768, 704), scales(g, 768)
    xs = [(bytes_(g, rows, 704), scales(g, rows)) for rows in (1, 9, 90, 2000)]
    plans = [pkg.Linear8(x.shape[0], 704, 768, out="float32") for x, _ in xs]
    want = [check(pkg, x, s, w, ws, "float32", plan=p) for (x, s), p in zip(xs, plans)]
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[torch.empty_like(v) for _ in range(6)] for v in want]
    torch.cuda.synchronize()
    for i in range(6):
        for (x, s), plan, stream, y in zip(xs, plans, streams, got):
            plan.forward(x, s, w, ws, y[i], stream=stream)
    for plan, stream in zip(plans, streams):
        plan.sync(stream)
        plan.close()
    assert all(torch.equal(y, v) for ys, v in zip(got, want) for y in ys)


def test_one_plan_many_calls(pkg):
    g = torch.Generator(device="cuda").manual_seed(4)
    k, n = 2000, 150
    w, ws = bytes_(g, n, k), scales(g, n)
    x, xs = bytes_(g, 200, k), scales(g, 200)
    with pkg.Linear8(200, k, n, out="float32") as plan:
        got = {}
        for rows in (200, 1, 40, 9, 200, 65, 1, 64, 40, 9, 0):
            if rows == 0:
                plan.forward(x[:0], xs[:0], w, ws, torch.empty(0, n, device="cuda"))
                plan.sync()
                continue
            y = check(pkg, x[:rows], xs[:rows], w, ws, "float32", plan=plan)
            assert rows not in got or torch.equal(got[rows], y)
            got[rows] = y
        # any number of rows gives a row the same bits
        assert torch.equal(got[200][:1], got[1]) and torch.equal(got[200][:40], got[40])


def test_streams_and_graphs(pkg):
    g = torch.Generator(device="cuda").manual_seed(5)
    for rows in (3, 50, 140):
        k, n = 512, 512
        w, ws = bytes_(g, n, k), scales(g, n)
        a, b = (torch.randn(rows, k, device="cuda", generator=g) for _ in range(2))
        q, s, y = (torch.empty(rows, k, device="cuda", dtype=torch.int8), torch.empty(rows, device="cuda"),
                   torch.empty(rows, n, device="cuda"))
        with pkg.Linear8(rows, k, n, out="float32") as plan:
            def step(v, stream=None):
                pkg.quantise(v, q, s, stream=stream)
                plan.forward(q, s, w, ws, y, stream=stream)
            held = a.clone()
            step(held)   # scratch is made here
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            want = {}
            for name, v in (("a", a), ("b", b)):
                step(v, side)
                plan.sync(side)
                want[name] = y.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(held, torch.cuda.current_stream())
            for name, v in (("b", b), ("a", a)):
                held.copy_(v)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(y, want[name])


def test_offsets_past_2_31(pkg):
    g = torch.Generator(device="cuda").manual_seed(6)
    k, n, far = 128, 40, (1 << 27) - 16
    big = torch.empty(far * n + k, device="cuda", dtype=torch.int8)
    w = bytes_(g, n, k)
    v = big.as_strided((n, k), (far, 1))
    v.copy_(w)
    for rows in (2, 70):
        x, xs, ws = bytes_(g, rows, k), scales(g, rows), scales(g, n)
        assert torch.equal(check(pkg, x, xs, v, ws, "float32"), check(pkg, x, xs, w, ws, "float32"))


# --------------------------------------------------------------- rounding

def round64(x):
    """The definition: 127 x is exact in float64, and so is its quotient where it
    lies at a half."""
    x = x.double()
    most = x.abs().max(dim=1, keepdim=True).values
    q = torch.round(127 * x / torch.where(most > 0, most, torch.ones_like(most)))
    return q.to(torch.int8), (most / 127).float()[:, 0]


def check_round(pkg, x, how="plain"):
    rows, n = x.shape
    q = torch.full((rows + 2, n + 3), 55, device="cuda", dtype=torch.int8)
    if how == "plain":
        out = torch.empty(rows, n, device="cuda", dtype=torch.int8)
    else:
        out = q[1:-1, 1:n + 1]
    scale = torch.full((rows + 2,), 55.0, device="cuda")
    pkg.quantise(x, out, scale[1:-1])
    torch.cuda.synchronize()
    want_q, want_scale = round64(x)
    assert torch.equal(out, want_q)
    assert torch.equal(scale[1:-1], want_scale)
    guard = q.clone()
    guard[1:-1, 1:n + 1] = 55
    assert bool((guard == 55).all()) and scale[0] == 55 and scale[-1] == 55


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 4096), (3, 5), (70, 33), (9, 128), (5, 1000), (4, 8192), (3, 8193),
                                    (2, 40000), (300, 64), (1, 100003)])
def test_rounding(pkg, dtype, rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    x = torch.randn(rows, n, device="cuda", generator=g).to(U.TYPES[dtype])
    check_round(pkg, x)
    check_round(pkg, x, "inside")
    x[:, n // 2] *= 30
    for how in ("turned", "slack", "odd", "apart"):
        check_round(pkg, lay(x, how), "inside")


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_rounding_next_to_a_half(pkg, dtype):
    """Values at (k + 1/2) / 127 of the largest and the nearest on both sides, for
    largest sizes of many kinds, 254 among them, where halves are met exactly."""
    t = U.TYPES[dtype]
    for most in (254.0, 127.0, 1.0, 3.0, 2.0 ** -10 * 254, 777.0, 0.1, 508.0, 33.3):
        most = float(torch.tensor(most).to(t))
        half = ((torch.arange(127, device="cuda", dtype=torch.float64) + 0.5) * most / 127).to(t)
        up, down = torch.nextafter(half, torch.full_like(half, 1e4)), torch.nextafter(half, torch.full_like(half, -1e4))
        row = torch.cat([half, up, down, torch.tensor([most], device="cuda", dtype=t)])
        check_round(pkg, torch.stack([row, -row, row.flip(0)]))


@pytest.mark.parametrize("most", [3.4e38, 1e-38, 1e-44, 2.0 ** -149, 1.1754944e-38, 2.0 ** 101, 2.0 ** -61])
def test_rounding_at_the_ends_of_the_range(pkg, most):
    g = torch.Generator(device="cuda").manual_seed(7)
    x = ((torch.rand(4, 300, device="cuda", generator=g, dtype=torch.float64) * 2 - 1) * most).float()
    x[:, 7] = most
    check_round(pkg, x)


def test_rounding_of_rows_without_a_scale(pkg):
    x = torch.randn(6, 100, device="cuda")
    x[1] = 0
    x[2, 5] = float("inf")
    x[2, 6] = -float("inf")
    x[3, 9] = float("nan")
    x[4, 1], x[4, 2] = float("nan"), float("inf")
    q, s = torch.empty(6, 100, device="cuda", dtype=torch.int8), torch.empty(6, device="cuda")
    pkg.quantise(x, q, s)
    torch.cuda.synchronize()
    assert s[1] == 0 and not bool(q[1].any())
    assert s[2] == float("inf") and q[2, 5] == 127 and q[2, 6] == -127 and int(q[2].abs().sum()) == 254
    assert bool(torch.isnan(s[3:5]).all()) and not bool(q[3:5].any())
    keep = [0, 5]
    want_q, want_s = round64(x[keep])
    assert torch.equal(q[keep], want_q) and torch.equal(s[keep], want_s)


def test_a_run_of_them(pkg):
    """As they are used: rounded activations through a row-parallel product split
    over four ranks, its float32 partials added up by a reduction, and experts on
    what comes out."""
    g = torch.Generator(device="cuda").manual_seed(8)
    rows, d, p = 6, 256, 4
    x = torch.randn(rows, d, device="cuda", generator=g)
    wide = torch.randn(d, d, device="cuda", generator=g) / 16
    w, ws = torch.empty(d, d, device="cuda", dtype=torch.int8), torch.empty(d, device="cuda")
    pkg.quantise(wide, w, ws)
    parts, total = [], torch.zeros(rows, d, device="cuda", dtype=torch.float64)
    for r in range(p):
        cut = slice(r * d // p, (r + 1) * d // p)
        q, s = torch.empty(rows, d // p, device="cuda", dtype=torch.int8), torch.empty(rows, device="cuda")
        pkg.quantise(x[:, cut], q, s)
        y = torch.empty(rows, d, device="cuda")
        with pkg.Linear8(rows, d // p, d, out="float32") as plan:
            plan.forward(q, s, w[:, cut], ws, y)
            plan.sync()
        parts.append(y.view(-1))
        total += product64(q, w[:, cut]) * s.double()[:, None] * ws.double()
    sums = [torch.empty_like(v) for v in parts]
    with pkg.Plan(p, rows * d, "float32") as plan:
        plan.allreduce(parts, sums)
        plan.sync()
    off = (sums[0].view(rows, d).double() - total).abs()
    assert bool((off <= 2.0 ** -21 * sum(v.view(rows, d).double().abs() for v in parts)).all())
    h = sums[0].view(rows, d).bfloat16()
    import test_gpu_experts as E
    _, router, w3, scale = E.make(rows, d, 64, 8, 8, "bfloat16", "int8", 3)
    E.check(pkg, h, router, w3, scale, 2, out="float32", weights="int8")
