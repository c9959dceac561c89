"""Experts on the GPU against the definition in 64 bits: sizes from one token,
expert and feature on, odd ones, every type, how the arrays lie, which experts
are here, ties and values without order, streams and graphs."""
import math

import pytest
import torch

import proj_util as U

pytestmark = pytest.mark.gpu

ROUND = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -23}


@pytest.fixture(scope="module")
def pkg():
    from paper_2109_12626_gb300 import build as B
    B.build()
    import paper_2109_12626_gb300 as pkg
    pkg.lib()
    return pkg


def layer64(x, router, w, scale, top, first, act, normalise, chosen=None):
    """y, chosen, share by the definition, and a bound of what a right kernel
    may be off by before it rounds y.

    Roundings, relative to the sum of the products' sizes: a float32 sum of k
    products (U.summed); the activation (U.EVAL); the hidden value kept to 21 bits
    and its products, 2^-20; the share, a few operations, 2^-20, and what the
    scores' own error makes of it."""
    x64, r64 = x.double(), router.double()
    scores = x64 @ r64.t()
    off = U.summed(x.shape[1]) * (x64.abs() @ r64.abs().t())
    order = torch.sort(scores, dim=1, descending=True, stable=True).indices[:, :top]
    if chosen is not None:
        # where scores are nearer than their error, either order is right
        chosen = chosen.long()
        assert all(len(set(row)) == top for row in chosen.tolist())
        gap = (scores.gather(1, order) - scores.gather(1, chosen)).abs()
        assert bool((gap <= off.max(dim=1, keepdim=True).values * 2).all())
        order = chosen
    picked = scores.gather(1, order)
    high = picked.max(dim=1, keepdim=True).values
    parts = torch.exp(picked - high)
    total = (parts if normalise else torch.exp(scores - high)).sum(dim=1, keepdim=True)
    share = parts / total
    share_off = share * (4 * off.max(dim=1, keepdim=True).values + 2.0 ** -20)
    y = torch.zeros_like(x64)
    bound = torch.zeros_like(x64)
    wide = [v.double() if s is None else v.double() * s.double()[:, :, None] for v, s in zip(w, scale)]
    for e in range(w[0].shape[0]):
        t, k = (order == first + e).nonzero(as_tuple=True)
        if len(t) == 0:
            continue
        a = x64[t]
        g, u = a @ wide[0][e].t(), a @ wide[1][e].t()
        sums = U.summed(x.shape[1]) + 2.0 ** -22
        g_off, u_off = sums * (a.abs() @ wide[0][e].abs().t()), sums * (a.abs() @ wide[1][e].abs().t())
        v = U.act64(act, g)
        h = v * u
        h_off = (U.LIPSCHITZ[act] * g_off + U.EVAL * v.abs()) * (u.abs() + u_off) + v.abs() * u_off + 2.0 ** -20 * h.abs()
        s, s_off = share[t, k][:, None], share_off[t, k][:, None]
        down = wide[2][e].abs().t()
        y.index_add_(0, t, s * (h @ wide[2][e].t()))
        bound.index_add_(0, t, s * (h_off @ down) + (s * (U.summed(h.shape[1]) + 2.0 ** -20) + s_off) * (h.abs() @ down))
    return y, order, share, bound + 2.0 ** -21 * y.abs(), share_off


def make(rows, d, h, total, local, dtype, weights, seed, pitch=0, place=0):
    """Inputs on the GPU; rows of the weights `pitch` elements further apart
    than they are long, the first `place` elements into its array."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = U.TYPES[dtype]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dt)

    def stack(n, k):
        if weights == "int8":
            v = torch.randint(-128, 128, (local, n, k), device="cuda", generator=g).to(torch.int8)
        else:
            v = normal(local, n, k, scale=k ** -0.5)
        if not pitch and not place:
            return v
        fill = 77 if weights == "int8" else float("nan")   # between the rows: never used
        whole = torch.full((place + local * n * (k + pitch) + 16,), fill, device="cuda", dtype=v.dtype)
        out = whole[place:place + local * n * (k + pitch)].view(local, n, k + pitch)[:, :, :k]
        out.copy_(v)
        return out

    w = [stack(h, d), stack(h, d), stack(d, h)]
    scale = [None] * 3
    if weights == "int8":
        scale = [(torch.rand(local, v.shape[1], device="cuda", generator=g) + 0.5) * v.shape[2] ** -0.5 / 64 for v in w]
    return normal(rows, d), normal(total, d, scale=d ** -0.5), w, scale


def run(pkg, x, router, w, scale, top, first=0, act="silu", out=None, weights=None, normalise=True, max_rows=None, plan=None):
    rows, d = x.shape
    dtype = str(x.dtype).split(".")[-1]
    out = out or dtype
    own = plan is None
    if own:
        plan = pkg.Experts(max_rows or rows, d, w[0].shape[1], router.shape[0], top, dtype, out=out,
                           weights=weights or dtype, act=act, first=first, local=w[0].shape[0], normalise=normalise)
    y = torch.full((rows + 2, d + 3), 7.0, device="cuda", dtype=U.TYPES[out])
    chosen = torch.full((rows, top), -5, device="cuda", dtype=torch.int32)
    share = torch.full((rows, top), -5.0, device="cuda")
    plan.forward(x, router, *w, y[1:-1, 1:d + 1], gate_scale=scale[0], up_scale=scale[1], down_scale=scale[2],
                 chosen=chosen, share=share)
    plan.sync()
    if own:
        plan.close()
    guard = y.clone()
    guard[1:-1, 1:d + 1] = 7.0
    assert bool((guard == 7.0).all()), "written outside the result"
    return y[1:-1, 1:d + 1].clone(), chosen, share


def check(pkg, x, router, w, scale, top, first=0, act="silu", out=None, weights=None, normalise=True, **more):
    y, chosen, share = run(pkg, x, router, w, scale, top, first, act, out, weights, normalise, **more)
    want, _, want_share, bound, share_off = layer64(x, router, w, scale, top, first, act, normalise, chosen)
    assert bool(((share.double() - want_share).abs() <= share_off).all())
    U.close("y", y, want, bound, out or str(x.dtype).split(".")[-1])
    return y, chosen, share


CASES = [  # rows, n_model, n_hidden, experts, top, dtype, weights, out
    (1, 64, 32, 4, 2, "bfloat16", None, None), (1, 1, 1, 1, 1, "bfloat16", None, None),
    (1, 4096, 512, 8, 2, "bfloat16", None, "float32"), (3, 200, 72, 8, 2, "float16", None, None),
    (8, 512, 256, 16, 4, "bfloat16", None, None), (9, 512, 256, 16, 4, "float16", None, "float32"),
    (17, 320, 96, 4, 1, "bfloat16", None, None), (33, 256, 128, 4, 3, "bfloat16", None, "float32"),
    (64, 128, 64, 4, 4, "bfloat16", None, None), (64, 256, 128, 128, 8, "float16", None, None),
    (40, 96, 40, 2, 2, "float16", None, "float32"), (5, 77, 33, 7, 3, "bfloat16", None, None),
    (5, 1001, 333, 12, 5, "float16", None, "float32"), (2, 2, 3, 40, 16, "bfloat16", None, None),
    (16, 72, 130, 512, 16, "bfloat16", None, None), (64, 65, 63, 200, 16, "float16", None, "float32"),
    (1, 1024, 2048, 64, 8, "bfloat16", "int8", None), (7, 192, 64, 8, 2, "float16", "int8", "float32"),
    (20, 129, 67, 6, 2, "bfloat16", "int8", "float32"), (64, 320, 192, 4, 2, "bfloat16", "int8", None),
    (33, 63, 257, 9, 1, "float16", "int8", None), (12, 31, 17, 33, 2, "bfloat16", "int8", None)]


@pytest.mark.parametrize("rows,d,h,total,top,dtype,weights,out", CASES)
def test_against_the_definition(pkg, rows, d, h, total, top, dtype, weights, out):
    x, router, w, scale = make(rows, d, h, total, total, dtype, weights, rows * 7 + d)
    check(pkg, x, router, w, scale, top, out=out, weights=weights, normalise=(rows + d) % 2 == 0)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid"])
def test_activations(pkg, act):
    x, router, w, scale = make(6, 160, 80, 5, 5, "bfloat16", None, 5)
    check(pkg, x, router, w, scale, 2, act=act, out="float32")


@pytest.mark.parametrize("weights", [None, "int8"])
@pytest.mark.parametrize("pitch,place", [(0, 8), (8, 0), (1, 0), (3, 5), (16, 1), (0, 3)])
def test_weights_at_any_address(pkg, weights, pitch, place):
    for rows, d, h in ((4, 96, 48), (11, 133, 71), (40, 64, 30)):
        x, router, w, scale = make(rows, d, h, 6, 6, "bfloat16", weights, 3 + pitch + place, pitch, place)
        check(pkg, x, router, w, scale, 2, out="float32", weights=weights)


def test_experts_one_matrix_for_all(pkg):
    x, router, w, scale = make(5, 96, 64, 6, 6, "bfloat16", None, 9)
    same = [v[2:3].expand(6, -1, -1) for v in w]
    check(pkg, x, router, same, scale, 3, out="float32")


def test_x_and_router_as_they_lie(pkg):
    x, router, w, scale = make(6, 136, 64, 10, 10, "float16", None, 4)
    turned = torch.empty(136, 6, device="cuda", dtype=x.dtype).t().copy_(x)
    r2 = torch.empty(136, 10, device="cuda", dtype=x.dtype).t().copy_(router)
    odd = torch.empty(6, 141, device="cuda", dtype=x.dtype)[:, 3:139].copy_(x)
    base = run(pkg, x, router, w, scale, 2)
    for a, b in ((turned, router), (x, r2), (odd, router), (turned, r2)):
        y, chosen, share = check(pkg, a, b, w, scale, 2)
        assert torch.equal(chosen, base[1])
    check(pkg, x[:1].expand(6, -1), router, w, scale, 2)


@pytest.mark.parametrize("first,local", [(0, 1), (3, 4), (15, 1), (8, 8)])
def test_some_experts_here(pkg, first, local):
    x, router, w, scale = make(21, 144, 64, 16, local, "bfloat16", None, first + 1)
    y, chosen, share = check(pkg, x, router, w, scale, 2, first=first, out="float32")
    here = ((chosen >= first) & (chosen < first + local)).any(dim=1)
    assert bool((y[~here] == 0).all())
    assert not bool(here.all())


def test_ranks_add_up(pkg):
    """Expert-parallel ranks' float32 results, and those of ranks that hold a slice
    of every expert, added up by a reduction, are the whole layer's."""
    x, router, w, scale = make(10, 128, 96, 12, 12, "bfloat16", None, 2)
    want, _, _, bound, _ = layer64(x, router, w, scale, 3, 0, "silu", True)
    for how in ("experts", "slices"):
        parts = []
        for r in range(4):
            if how == "experts":
                mine, first, local, h = [v[3 * r:3 * r + 3] for v in w], 3 * r, 3, 96
            else:
                mine, first, local, h = [w[0][:, 24 * r:24 * r + 24], w[1][:, 24 * r:24 * r + 24], w[2][:, :, 24 * r:24 * r + 24]], 0, 12, 24
            y = torch.empty(10, 128, device="cuda")
            with pkg.Experts(10, 128, h, 12, 3, "bfloat16", out="float32", first=first, local=local) as plan:
                plan.forward(x, router, *mine, y)
                plan.sync()
            parts.append(y.reshape(-1))
        sums = [torch.empty_like(p) for p in parts]
        with pkg.Plan(4, 1280, "float32") as plan:
            plan.allreduce(parts, sums)
            plan.sync()
        U.close("sum", sums[3].view(10, 128), want, bound * 2 + 2.0 ** -21 * want.abs(), "float32")


def test_none_here_gives_zeros(pkg):
    x, router, w, scale = make(4, 64, 32, 8, 2, "bfloat16", None, 6)
    x = x.abs()
    router = -router.abs()
    router[:2] = router[2:].abs().max() * 4
    y, chosen, _ = run(pkg, x, router, w, scale, 2, first=6)
    assert bool((chosen < 2).all()) and bool((y == 0).all())


def test_equal_scores_take_the_lower_number(pkg):
    x, router, w, scale = make(9, 64, 32, 70, 70, "bfloat16", None, 8)
    router = router[:1].expand(70, -1)
    _, chosen, share = run(pkg, x, router, w, scale, 5)
    assert torch.equal(chosen, torch.arange(5, device="cuda", dtype=torch.int32).expand(9, 5))
    assert torch.allclose(share, torch.full_like(share, 0.2), rtol=2.0 ** -20, atol=0)
    _, chosen, _ = run(pkg, torch.zeros_like(x) * -1.0, router, w, scale, 5)   # 0 and -0 alike
    assert torch.equal(chosen, torch.arange(5, device="cuda", dtype=torch.int32).expand(9, 5))


def test_not_a_number_stays_in_its_row(pkg):
    x, router, w, scale = make(10, 96, 48, 8, 8, "bfloat16", None, 10)
    _, chosen, _ = run(pkg, x, router, w, scale, 2, out="float32")
    want, _, _, bound, _ = layer64(x, router, w, scale, 2, 0, "silu", True, chosen)
    for bad in (float("nan"), float("inf")):
        v = x.clone()
        v[3, 5] = bad
        y, c, s = run(pkg, v, router, w, scale, 2, out="float32")
        keep = torch.arange(10, device="cuda") != 3
        # where the long sums are cut depends on what all tokens chose, and with it
        # the order of a sum's additions, which the bound allows for
        U.close("y", y[keep], want[keep], bound[keep], "float32")
        assert torch.equal(c[keep], chosen[keep])
        assert not bool(torch.isfinite(y[3]).any())
    # an expert that no token chose may hold anything
    _, c, _ = run(pkg, x[:2], router, w, scale, 2)
    unused = [e for e in range(8) if e not in c.flatten().tolist()][0]
    v = [t.clone() for t in w]
    for t in v:
        t[unused] = float("nan")
    assert bool(torch.isfinite(run(pkg, x[:2], router, v, scale, 2)[0]).all())


def test_large_hidden_values_of_float16(pkg):
    """Hidden values beyond float16's range are held in float32."""
    x, router, w, scale = make(3, 128, 64, 4, 4, "float16", None, 12)
    w[0], w[1], w[2] = w[0] * 300, w[1] * 300, w[2] / 8192
    assert layer64(x, router, w, scale, 2, 0, "relu", True)[0].abs().max() < 60000
    hidden = torch.relu(x.double() @ w[0][0].double().t()) * (x.double() @ w[1][0].double().t())
    assert hidden.abs().max() > 65504
    check(pkg, x, router, w, scale, 2, act="relu", out="float32")


def test_one_plan_many_calls(pkg):
    """Fewer rows than the plan takes, back to back, the same bits each time; what
    one call left does not show in the next."""
    x, router, w, scale = make(30, 264, 96, 16, 16, "bfloat16", None, 13)
    with pkg.Experts(40, 264, 96, 16, 4, "bfloat16", out="float32") as plan:
        got = {}
        for rows in (30, 1, 7, 30, 16, 1, 30, 7):
            y, c, s = run(pkg, x[:rows], router, w, scale, 4, out="float32", plan=plan)
            if rows in got:
                assert torch.equal(y, got[rows])
            got[rows] = y
            want, _, _, bound, _ = layer64(x[:rows], router, w, scale, 4, 0, "silu", True, c)
            U.close("y", y, want, bound, "float32")
        none = torch.empty(0, 264, device="cuda", dtype=torch.bfloat16)
        plan.forward(none, router, *w, torch.empty(0, 264, device="cuda"))
        plan.sync()


def test_streams_and_graphs(pkg):
    x, router, w, scale = make(12, 256, 128, 16, 16, "bfloat16", None, 14)
    with pkg.Experts(12, 256, 128, 16, 4, "bfloat16") as plan:
        want = run(pkg, x, router, w, scale, 4, plan=plan)[0]
        y = torch.empty_like(x)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        plan.forward(x, router, *w, y, stream=side)
        plan.sync(side)
        assert torch.equal(y, want)
        other = make(12, 256, 128, 16, 16, "bfloat16", None, 15)[0]
        held = other.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.forward(held, router, *w, y, stream=torch.cuda.current_stream())
            plan.forward(y, router, *w, held, stream=torch.cuda.current_stream())
        for inputs in (other, x):
            held.copy_(inputs)
            graph.replay()
            torch.cuda.synchronize()
            first = run(pkg, inputs, router, w, scale, 4, plan=plan)[0]
            second = run(pkg, first, router, w, scale, 4, plan=plan)[0]
            assert torch.equal(y, first) and torch.equal(held, second)


def test_split_sums_and_many_blocks(pkg):
    """Few units with long sums, whose parts several CTAs form, and more units
    than CTAs."""
    for rows, d, h, total, top in ((1, 8192, 64, 4, 1), (2, 64, 8192, 2, 1), (1, 4096, 4096, 2, 1), (3, 2048, 1024, 64, 16)):
        x, router, w, scale = make(rows, d, h, total, total, "bfloat16", None, d + h)
        check(pkg, x, router, w, scale, top, out="float32")


def test_offsets_past_2_31(pkg):
    """Experts whose weights lie more than 2^31 elements into their array."""
    d, h, total = 128, 64, 3
    far = (1 << 31) + 64
    x, router, w, scale = make(4, d, h, total, total, "bfloat16", None, 16)
    whole = torch.empty(far * 2 + d * h, device="cuda", dtype=torch.bfloat16)
    for v in w:
        n, k = v.shape[1:]
        s = whole.as_strided((total, n, k), (far, k, 1))
        s.copy_(v)
        y, c, _ = run(pkg, x, router, [s if q is v else q for q in w], scale, 2, out="float32")
        want, _, _, bound, _ = layer64(x, router, w, scale, 2, 0, "silu", True, c)
        U.close("y", y, want, bound, "float32")


def test_refusals(pkg):
    with pytest.raises(pkg.DpdrError):
        pkg.Experts(65, 64, 32, 4, 2)
    x, router, w, scale = make(4, 64, 32, 4, 4, "bfloat16", None, 1)
    y = torch.empty_like(x)
    with pkg.Experts(4, 64, 32, 4, 2) as plan:
        with pytest.raises(ValueError):
            plan.forward(x, router, w[0], w[1], w[2].transpose(1, 2), y)
        with pytest.raises(pkg.DpdrError):
            plan.forward(x, router, *w, x)                 # a result over an input
        with pytest.raises(pkg.DpdrError):
            plan.forward(x, router, w[0], w[1], w[2].transpose(1, 2).contiguous().transpose(1, 2), y)
        with pytest.raises(TypeError):
            plan.forward(x.half(), router, *w, y)
        with pytest.raises(pkg.DpdrError):                 # scales without 8-bit weights
            plan.forward(x, router, *w, y, gate_scale=torch.ones(4, 32, device="cuda"))
        with pytest.raises(ValueError):
            plan.forward(x, router, *w, y, chosen=torch.empty(2, 4, device="cuda", dtype=torch.int32).t())
        five = torch.cat([x, x[:1]])
        with pytest.raises(pkg.DpdrError):
            plan.forward(five, router, *w, torch.empty_like(five))
    with pkg.Experts(4, 64, 32, 4, 2, weights="int8") as plan:
        w8 = [v.to(torch.int8) for v in w]
        with pytest.raises(pkg.DpdrError):                 # and the other way round
            plan.forward(x, router, *w8, y)


def test_two_plans_on_two_streams(pkg):
    """Calls of different plans may overlap: each has scratch of its own."""
    cases = [make(rows, 320, 160, 24, 24, "bfloat16", weights, rows) for rows, weights in ((1, None), (30, None), (8, "int8"))]
    plans = [pkg.Experts(c[0].shape[0], 320, 160, 24, 4, out="float32", weights=w) for c, w in zip(cases, (None, None, "int8"))]
    want = [run(pkg, *c, 4, out="float32", plan=p)[0] for c, p in zip(cases, plans)]
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[torch.empty_like(w) for _ in range(6)] for w in want]
    torch.cuda.synchronize()
    for i in range(6):
        for (x, router, w, scale), plan, stream, y in zip(cases, plans, streams, got):
            plan.forward(x, router, *w, y[i], gate_scale=scale[0], up_scale=scale[1], down_scale=scale[2], stream=stream)
    for plan, stream in zip(plans, streams):
        plan.sync(stream)
        plan.close()
    assert all(torch.equal(y, w) for ys, w in zip(got, want) for y in ys)


@pytest.mark.parametrize("ranks,tokens", [(1, 3), (4, 1), (4, 40), (2, 64)])
def test_the_example_runs(ranks, tokens):
    """examples/expert_parallel_tokens.py: sums of some hundred products in float32,
    2^-24 a step at most, of values of one size."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import expert_parallel_tokens as example
    block = example.SplitTokens(ranks, tokens, 256, 128, 8, 2)
    x = torch.randn(tokens, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    for _ in range(2):
        block.forward(x)
        block.sync()
    errors = example.worst(block, x)
    assert max(errors.values()) < 512 * 2.0 ** -24, errors
    block.close()
