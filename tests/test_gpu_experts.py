"""GPU: the operators of a mixture-of-experts layer against plain 64-bit forms.

Tolerances.  u is the unit roundoff of the output's type (2^-8 BF16, 2^-11 FP16,
2^-24 FP32): the one rounding of an output costs u |y|; E = 2^-24 is FP32's.
Chosen experts, plans, INT32 sums and carriers are exact.
"""
import numpy as np
import pytest

from tests._cases import W8_DENSE, W8_ROUTED, say

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0**-8, "fp16": 2.0**-11, "fp32": 2.0**-24}
E = 2.0**-24
TINY = 2.0**-24  # smallest subnormal of FP16


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2608_06763_amd as cq
    cq.lib()
    return torch


def _cq():
    import paper_2608_06763_amd as cq
    return cq


def _dtype(torch, name):
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def _rand(torch, seed, *shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(_dtype(torch, dtype)).cuda()


def _int8(torch, seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-128, 128, shape, generator=g, dtype=torch.int8).cuda()


def _f64(t):
    return t.detach().cpu().double().numpy()


def _within(got, ref, bound, what):
    got = _f64(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), what
    off = np.abs(got - ref) - bound
    assert (off <= 0).all(), f"{what}: {np.max(off)} over the bound at {np.unravel_index(np.argmax(off), off.shape)}"


# ---------------------------------------------------------------- routing


def _route_ref(l, top, scoring="softmax", bias=None, groups=1, kept_groups=1, group_top=1, renormalize=True, scale=1.0,
               live=None):
    """One token at a time, from the definition."""
    tokens, experts = l.shape
    chosen, weights = np.full((tokens, top), -1, np.int64), np.zeros((tokens, top))
    size = experts // groups
    for t in range(tokens if live is None else max(0, min(live, tokens))):
        may = [e for e in range(experts) if l[t, e] > -np.inf]
        score = {}
        if may and scoring == "softmax":
            m = max(l[t, e] for e in may)
            part = {e: 1.0 if l[t, e] == m else np.exp(l[t, e] - m) for e in may}
            score = {e: v / sum(part.values()) for e, v in part.items()}
        elif may:
            score = {e: 1.0 / (1.0 + np.exp(-l[t, e])) for e in may}
        # without a bias the order is that of the logits, without their rounding to scores
        c = {e: l[t, e] if bias is None else score[e] + bias[e] for e in may}
        c = {e: v for e, v in c.items() if v > -np.inf}
        if kept_groups < groups:
            value = {}
            adds = c if bias is not None or group_top == 1 else score
            for g in range(groups):
                best = sorted((adds[e] for e in c if e // size == g), reverse=True)[:group_top]
                if best:
                    value[g] = sum(best)
            kept = sorted(value, key=lambda g: (-value[g], g))[:kept_groups]
            c = {e: v for e, v in c.items() if e // size in kept}
        pick = sorted(c, key=lambda e: (-c[e], e))[:top]
        w = np.array([score[e] for e in pick])
        if renormalize and pick:
            if scoring == "softmax":
                # from the chosen alone, which all scores may be far above
                m = max(l[t, e] for e in pick)
                w = np.array([1.0 if l[t, e] == m else np.exp(l[t, e] - m) for e in pick])
            if w.sum() > 0:
                w = w / w.sum()
        chosen[t, :len(pick)], weights[t, :len(pick)] = pick, w * scale
    return chosen, weights


def _plan_ref(chosen, experts):
    flat = chosen.ravel()
    taken = np.flatnonzero(flat >= 0)
    order = taken[np.argsort(flat[taken], kind="stable")]
    ends = np.cumsum(np.concatenate([[0], np.bincount(flat[taken], minlength=experts)]))
    return np.concatenate([ends, order, np.full(flat.size - taken.size, -1)])


def _check_route(torch, logits, top, what, **kw):
    cq = _cq()
    got = cq.cq_route(logits, top, **kw)
    opt = {k: v for k, v in kw.items() if k not in ("bias", "live", "stream")}
    if kw.get("bias") is not None:
        opt["bias"] = _f64(kw["bias"])
    if kw.get("live") is not None:
        opt["live"] = int(kw["live"].item())
    with np.errstate(over="ignore"):
        chosen, weights = _route_ref(_f64(logits), top, **opt)
    assert np.array_equal(got[0].cpu().numpy(), chosen), what
    assert np.array_equal(got[2].cpu().numpy(), _plan_ref(chosen, logits.shape[1])), what
    # exponents of differences up to 64 lose 64 E each, which doubles in a quotient; sums
    # of up to 1024 terms in a tree of ten, the quotient, exp and scale some units more
    _within(got[1], weights, 160.0 * E * np.abs(weights) + 2.0**-126, what)
    return got


ROUTES = [
    dict(), dict(scoring="sigmoid"), dict(renormalize=False, scale=2.5), dict(scoring="sigmoid", renormalize=False),
    dict(bias=1), dict(scoring="sigmoid", bias=1, scale=0.5), dict(bias=1, renormalize=False),
]


@pytest.mark.parametrize("tokens,experts,top", [(1, 1, 1), (1, 8, 2), (3, 7, 7), (1, 128, 8), (5, 60, 4), (70, 64, 6),
                                                (130, 65, 1), (33, 160, 32), (700, 256, 8), (9, 384, 12), (17, 1000, 10),
                                                (2, 1024, 32), (1500, 40, 3), (64, 512, 15),
                                                (65, 512, 15), (65, 512, 16), (32, 513, 8), (33, 240, 9), (2000, 128, 2), (17000, 12, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_route(torch_dev, tokens, experts, top, dtype):
    torch = torch_dev
    for n, f in enumerate(ROUTES):
        say("route", tokens, experts, top, dtype, f)
        logits = _rand(torch, 100 + n, tokens, experts, dtype=dtype, scale=2.0)
        kw = dict(f)
        if f.get("bias"):
            kw["bias"] = _rand(torch, 200 + n, experts, dtype="fp32", scale=0.1)
        _check_route(torch, logits, top, (n, f), **kw)


@pytest.mark.parametrize("experts,groups,kept,top", [(8, 2, 1, 3), (16, 8, 3, 6), (64, 8, 4, 8), (256, 8, 4, 8),
                                                     (160, 5, 2, 6), (100, 50, 20, 12), (64, 64, 9, 9), (1024, 16, 3, 32),
                                                     (60, 4, 3, 5), (512, 4, 4, 10), (72, 8, 1, 9), (16, 16, 5, 5),
                                                     (5, 5, 2, 2), (64, 4, 1, 20)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_groups(torch_dev, experts, groups, kept, top, scoring):
    # the last one keeps fewer experts than it asks for
    torch = torch_dev
    for n, (tokens, biased, group_top, dtype) in enumerate([(1, 1, 2, "bf16"), (37, 0, 1, "bf16"), (37, 0, 2, "fp32"),
                                                            (150, 1, 1, "fp16"), (150, 1, 2, "bf16")]):
        say("route groups", experts, groups, kept, top, scoring, tokens, biased, group_top, dtype)
        logits = _rand(torch, 300 + n, tokens, experts, dtype=dtype, scale=1.5)
        bias = _rand(torch, 310 + n, experts, dtype="fp32", scale=0.1) if biased else None
        _check_route(torch, logits, top, n, scoring=scoring, bias=bias, groups=groups, kept_groups=kept,
                     group_top=group_top, scale=2.5)


@pytest.mark.parametrize("experts,groups,kept", [(8, 1, 1), (64, 8, 3), (100, 1, 1), (256, 16, 5), (1024, 1, 1)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_ties_go_to_the_lowest_index(torch_dev, experts, groups, kept, scoring):
    torch = torch_dev
    for n, biased in enumerate([False, True]):
        for levels in (1, 2, 5):
            say("route ties", experts, groups, scoring, biased, levels)
            g = torch.Generator().manual_seed(7 * n + levels)
            logits = torch.randint(0, levels, (40, experts), generator=g).to(torch.bfloat16).cuda() - 1.0
            logits[::2] *= -1.0  # zeros of both signs
            bias = (torch.randint(0, 2, (experts,), generator=g) * 0.25).cuda() if biased else None
            for group_top in (1, 2):
                _check_route(torch, logits, min(8, experts), levels, scoring=scoring, bias=bias, groups=groups,
                             kept_groups=kept, group_top=group_top)


def test_route_neighbours_closer_than_fp32(torch_dev):
    # scores that differ by less than FP32's step of one, on top of a bias that hides them
    torch = torch_dev
    base = torch.linspace(-3.0, 3.0, 128).repeat(64, 1)
    step = torch.arange(64)[:, None] * torch.randint(-3, 4, (64, 128), generator=torch.Generator().manual_seed(5))
    logits = (base + step * 2.0**-21).cuda()
    for scoring in ("softmax", "sigmoid"):
        score = torch.softmax(base.double(), 1) if scoring == "softmax" else torch.sigmoid(base.double())
        bias = (1.0 - score[0]).float().cuda()  # all choices near one
        for opt in (dict(), dict(groups=8, kept_groups=3, group_top=2), dict(groups=16, kept_groups=3)):
            say("route near", scoring, opt)
            _check_route(torch, logits, 8, scoring, scoring=scoring, bias=bias, **opt)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_route_of_infinities_and_nan(torch_dev, scoring, dtype):
    torch = torch_dev
    inf, nan = float("inf"), float("nan")
    low = torch.finfo(_dtype(torch, dtype)).min
    logits = _rand(torch, 40, 12, 96, dtype=dtype)
    logits[0] = -inf
    logits[1] = nan
    logits[2, ::2] = -inf
    logits[3, 1::3] = nan
    logits[4, 5], logits[4, 50] = inf, inf
    logits[5] = low
    logits[6] = -inf
    logits[6, 95] = 1.0
    logits[7, :94] = nan
    logits[8, 3:] = low
    logits[9] = inf
    logits[10, 10:] = -60.0
    bias = _rand(torch, 41, 96, dtype="fp32", scale=0.1)
    odd = bias.clone()
    odd[:40], odd[40], odd[41] = -inf, nan, inf
    for n, opt in enumerate([dict(), dict(renormalize=False), dict(bias=bias), dict(bias=odd),
                             dict(bias=odd, groups=12, kept_groups=3, group_top=2),
                             dict(groups=12, kept_groups=3, group_top=2), dict(groups=12, kept_groups=2),
                             dict(groups=3, kept_groups=2, bias=bias)]):
        say("route odd values", scoring, dtype, n)
        _check_route(torch, logits, 6, n, scoring=scoring, **opt)


@pytest.mark.parametrize("tokens,live", [(1, 0), (1, 1), (50, 0), (50, 17), (50, 50), (50, 99), (50, -3), (900, 333)])
def test_route_tokens_that_do_not_count(torch_dev, tokens, live):
    torch = torch_dev
    logits = _rand(torch, 50, tokens, 48, dtype="bf16")
    logits[max(0, live):] = float("nan")
    for bias in (None, _rand(torch, 51, 48, dtype="fp32")):
        _check_route(torch, logits, 5, live, bias=bias, live=torch.tensor([live], dtype=torch.int32, device="cuda"))


def test_route_of_strided_logits_and_given_outputs(torch_dev):
    torch, cq = torch_dev, _cq()
    wide = _rand(torch, 60, 77, 200, dtype="fp32")
    outs = dict(chosen=torch.empty((77, 4), dtype=torch.int32, device="cuda"),
                weights=torch.empty((77, 4), device="cuda"),
                plan=torch.empty((64 + 1 + 77 * 4,), dtype=torch.int32, device="cuda"))
    got = _check_route(torch, wide[:, 8:72], 4, "strided", **{k: v for k, v in outs.items() if k == "none"})
    again = cq.cq_route(wide[:, 8:72], 4, **outs)
    for a, b, name in zip(got, again, outs):
        assert b is outs[name] and torch.equal(a, b)


@pytest.mark.parametrize("experts", [1, 2, 64, 100, 1000, 1024])
@pytest.mark.parametrize("routes", [1, 2, 63, 64, 65, 255, 1000, 1024, 1025, 4096, 4097, 5000, 70001, 300000, 700003])
def test_route_plan(torch_dev, experts, routes):
    torch, cq = torch_dev, _cq()
    say("plan", experts, routes)
    g = torch.Generator().manual_seed(routes)
    maps = [torch.randint(0, experts, (routes,), generator=g), torch.randint(-2, experts + 2, (routes,), generator=g),
            torch.full((routes,), experts - 1), torch.full((routes,), -1),
            torch.where(torch.rand(routes, generator=g) < 0.9, 0, torch.randint(0, experts, (routes,), generator=g))]
    for n, m in enumerate(maps):
        plan = torch.full((experts + 1 + routes,), -77, dtype=torch.int32, device="cuda")
        cq.cq_route_plan(m.to(torch.int32).cuda(), experts, plan=plan)
        flat = m.numpy()
        assert np.array_equal(plan.cpu().numpy(), _plan_ref(np.where((flat >= 0) & (flat < experts), flat, -1), experts)), n


# ---------------------------------------------------------------- products


def _product_ref(x8, dx, w8, dw, bias):
    """(y, magnitude before the bias, |bias|), the sums exact: below 2^53 in FP64."""
    p = _f64(x8) @ _f64(w8).T
    y = p * _f64(dx)[:, None] * _f64(dw)
    b = np.zeros_like(y) if bias is None else np.broadcast_to(_f64(bias), y.shape)
    return y + b, np.abs(y), np.abs(b)


def _product_bound(ref, mag, b, dtype):
    # the sum to FP32, dx dw, their product: three roundings; the bias one more
    return U[dtype] * np.abs(ref) * (1.0 + 4.0 * E) + 4.0 * E * (mag + b) + TINY


def _scales(torch, seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(shape, generator=g) * 0.02 + 0.001).cuda()


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 48, 64, 65, 100, 128, 129, 257, 400])
@pytest.mark.parametrize("n,k", [(1, 16), (3, 48), (16, 112), (17, 128), (40, 144), (100, 256), (128, 1040), (130, 512),
                                 (257, 272), (600, 2048), (64, 8208)])
def test_product(torch_dev, rows, n, k):
    torch, cq = torch_dev, _cq()
    x8, w8 = _int8(torch, rows + k, rows, k), _int8(torch, n + k, n, k)
    dx, dw = _scales(torch, 1, rows), _scales(torch, 2, n)
    for dtype in ("bf16", "fp16", "fp32"):
        for biased in (False, True):
            say("product", rows, n, k, dtype, biased)
            bias = _rand(torch, 3, n, dtype=dtype) if biased else None
            # what lies behind the output stays
            room = torch.full((rows * n + 64,), 7.0, dtype=_dtype(torch, dtype), device="cuda")
            got = cq.cq_gemm_w8(x8, dx, w8, dw, bias=bias, out=room[:rows * n].view(rows, n))
            ref, mag, b = _product_ref(x8, dx, w8, dw, bias)
            _within(got, ref, _product_bound(ref, mag, b, dtype), (rows, n, k, dtype, biased))
            assert bool((room[rows * n:] == 7.0).all())


@pytest.mark.parametrize("rows,n", [(1, 5), (20, 33), (70, 40), (130, 129), (300, 300)])
def test_product_of_the_longest_rows_and_largest_values(torch_dev, rows, n):
    torch, cq = torch_dev, _cq()
    k = 131056
    x8 = torch.full((rows, k), -128, dtype=torch.int8, device="cuda")
    w8 = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    x8[1::2], w8[::3] = 127, 127
    w8[:, -16:] = 1  # the last codes count
    one = torch.ones((max(rows, n),), device="cuda")
    y = cq.cq_gemm_w8(x8, one[:rows], w8, one[:n], y_dtype=torch.float32)
    ref = _f64(x8[:2]) @ _f64(w8[:2]).T if rows > 1 else _f64(x8) @ _f64(w8[:2]).T
    want = np.array([[ref[i % 2, 0 if j % 3 == 0 else 1] for j in range(n)] for i in range(rows)])
    assert np.abs(want).max() == (k - 16) * 128**2 - 16 * 128 > 2**31 - 2**20
    assert np.array_equal(_f64(y), want.astype(np.float32).astype(np.float64))


def _routed_ref(x8, dx, w8, dw, chosen, fan, bias):
    flat = chosen.cpu().numpy().ravel()
    experts, n, _ = w8.shape
    x, d = _f64(x8), _f64(dx)
    ref, mag, b = (np.zeros((flat.size, n)) for _ in range(3))
    for e in range(experts):
        r = np.flatnonzero(flat == e)
        if r.size:
            y = (x[r // fan] @ _f64(w8[e]).T) * d[r // fan][:, None] * _f64(dw[e])
            mag[r] = np.abs(y)
            if bias is not None:
                b[r] = np.abs(_f64(bias[e]))
                y = y + _f64(bias[e])
            ref[r] = y
    return ref, mag, b, (flat >= 0) & (flat < experts)


@pytest.mark.parametrize("experts,tokens,top,n,k", [
    (1, 1, 1, 40, 64), (8, 1, 2, 100, 128), (64, 1, 8, 64, 512), (64, 3, 8, 33, 272), (16, 61, 6, 48, 144),
    (5, 40, 3, 130, 256), (3, 200, 2, 129, 112), (40, 300, 4, 64, 64), (128, 9, 8, 20, 1040), (2, 700, 1, 257, 160),
    (1000, 30, 5, 16, 32), (4, 129, 4, 260, 384)])
@pytest.mark.parametrize("fan", [True, False])
def test_routed_product(torch_dev, experts, tokens, top, n, k, fan):
    torch, cq = torch_dev, _cq()
    g = torch.Generator().manual_seed(experts * tokens)
    w8, dw = _int8(torch, 1, experts, n, k), _scales(torch, 2, experts, n)
    rows = tokens if fan else tokens * top
    x8, dx = _int8(torch, 3, rows, k), _scales(torch, 4, rows)
    maps = [torch.randint(0, experts, (tokens, top), generator=g), torch.randint(-1, experts + 1, (tokens, top), generator=g),
            torch.full((tokens, top), experts // 2), torch.full((tokens, top), -1)]
    for m, dtype, biased in zip(maps, ("bf16", "fp32", "fp16", "bf16"), (False, True, True, False)):
        say("routed", experts, tokens, top, n, k, fan, dtype, biased)
        chosen = m.to(torch.int32).cuda()
        plan = cq.cq_route_plan(chosen, experts)
        bias = _rand(torch, 5, experts, n, dtype=dtype) if biased else None
        out = torch.full((tokens * top, n), 77.0, dtype=_dtype(torch, dtype), device="cuda")
        got = cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=top if fan else 1, bias=bias, out=out)
        ref, mag, b, there = _routed_ref(x8, dx, w8, dw, chosen, top if fan else 1, bias)
        assert bool((got.cpu()[torch.from_numpy(~there)] == 77.0).all())
        at = np.flatnonzero(there)
        _within(got[torch.from_numpy(at).cuda()], ref[at], _product_bound(ref, mag, b, dtype)[at], "routed")


def _check_on_device(torch, got, x8, dx, w8, dw, bias, dtype, what):
    """The same bound as above, formed on the device in FP64 (its sums are exact too)."""
    mag = (x8.double() @ w8.double().t()) * dx.double()[:, None] * dw.double()
    b = torch.zeros_like(mag) if bias is None else bias.double().expand_as(mag)
    ref = mag + b
    off = (got.double() - ref).abs() - (U[dtype] * ref.abs() * (1.0 + 4.0 * E) + 4.0 * E * (mag.abs() + b.abs()) + TINY)
    assert bool((off <= 0).all()), (what, float(off.max()))


@pytest.mark.parametrize("rows,n,k", [(9, 28667, 144), (16, 40000, 1040), (31, 28667, 272), (64, 28667, 144), (65, 30000, 128),
                                      (128, 28667, 656), (129, 20001, 144), (256, 28667, 400), (383, 20008, 16), (1000, 28667, 144),
                                      (1025, 16385, 528), (2500, 8191, 1168)])
def test_product_of_many_tiles(torch_dev, rows, n, k):
    torch, cq = torch_dev, _cq()
    x8, w8 = _int8(torch, rows + k, rows, k), _int8(torch, n + k, n, k)
    dx, dw = _scales(torch, 1, rows), _scales(torch, 2, n)
    for dtype, biased in (("bf16", False), ("fp16", True), ("fp32", True)):
        say("product of many tiles", rows, n, k, dtype, biased)
        bias = _rand(torch, 3, n, dtype=dtype) if biased else None
        room = torch.full((rows * n + 64,), 7.0, dtype=_dtype(torch, dtype), device="cuda")
        got = cq.cq_gemm_w8(x8, dx, w8, dw, bias=bias, out=room[:rows * n].view(rows, n))
        _check_on_device(torch, got, x8, dx, w8, dw, bias, dtype, (rows, n, k, dtype))
        assert bool((room[rows * n:] == 7.0).all())


@pytest.mark.parametrize("experts,tokens,top,n,k", [(64, 400, 4, 1001, 272), (64, 900, 4, 1000, 144), (32, 1000, 4, 1703, 400),
                                                    (16, 3000, 3, 1704, 144), (8, 60, 2, 8000, 512), (128, 60, 8, 700, 1040),
                                                    (3, 5000, 1, 5000, 48)])
@pytest.mark.parametrize("fan", [True, False])
def test_routed_product_of_many_tiles(torch_dev, experts, tokens, top, n, k, fan):
    torch, cq = torch_dev, _cq()
    g = torch.Generator().manual_seed(experts * tokens)
    w8, dw = _int8(torch, 1, experts, n, k), _scales(torch, 2, experts, n)
    rows = tokens if fan else tokens * top
    x8, dx = _int8(torch, 3, rows, k), _scales(torch, 4, rows)
    # some experts far more in demand than others, some routes of none
    chosen = (torch.rand((tokens, top), generator=g) ** 2 * (experts + 1)).long() - 1
    flat = chosen.flatten().cuda()
    plan = cq.cq_route_plan(chosen.to(torch.int32).cuda(), experts)
    for dtype, biased in (("bf16", True), ("fp32", False)):
        say("routed product of many tiles", experts, tokens, top, n, k, fan, dtype)
        bias = _rand(torch, 5, experts, n, dtype=dtype) if biased else None
        out = torch.full((tokens * top, n), 77.0, dtype=_dtype(torch, dtype), device="cuda")
        cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=top if fan else 1, bias=bias, out=out)
        assert bool((out[flat < 0] == 77.0).all())
        for e in range(experts):
            r = (flat == e).nonzero()[:, 0]
            at = r // top if fan else r
            if r.numel():
                _check_on_device(torch, out[r], x8[at], dx[at], w8[e], dw[e], None if bias is None else bias[e], dtype, e)


def test_routed_product_equals_the_dense_one(torch_dev):
    # every route with the one expert: the same numbers, whatever the tiles
    torch, cq = torch_dev, _cq()
    for rows in (1, 30, 200):
        x8, dx = _int8(torch, 1, rows, 400), _scales(torch, 2, rows)
        w8, dw = _int8(torch, 3, 1, 70, 400), _scales(torch, 4, 1, 70)
        plan = cq.cq_route_plan(torch.zeros((rows,), dtype=torch.int32, device="cuda"), 1)
        assert torch.equal(cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan), cq.cq_gemm_w8(x8, dx, w8[0], dw[0]))


def test_routed_product_of_plans_that_are_none(torch_dev):
    # offsets and routes outside the call's buffers reach nothing outside them
    torch, cq = torch_dev, _cq()
    experts, routes, n, k = 5, 300, 40, 64
    x8, dx = _int8(torch, 1, 150, k), _scales(torch, 2, 150)
    w8, dw = _int8(torch, 3, experts, n, k), _scales(torch, 4, experts, n)
    room = torch.full((routes + 40, n), 77.0, dtype=torch.bfloat16, device="cuda")
    big = 2**31 - 1
    for offsets in ([0, big, 0, big, -5, big], [big] * 6, [-big] * 6, [0, 60, 120, 180, 240, big], [300, 10, 300, 0, 300, 0]):
        for order in (-1, big, routes, 5):
            say("plan", offsets, order)
            plan = torch.tensor(offsets + [order] * routes, dtype=torch.int32, device="cuda")
            cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=2, out=room[20:20 + routes])
            torch.cuda.synchronize()
            assert bool((room[:20] == 77.0).all()) and bool((room[20 + routes:] == 77.0).all())


def test_product_offsets_past_32_bits(torch_dev):
    torch, cq = torch_dev, _cq()
    # the last expert's weights lie behind 4 GiB
    experts, n, k = 1024, 1040, 4096
    w8 = torch.empty((experts, n, k), dtype=torch.int8, device="cuda")
    w8[-1] = _int8(torch, 1, n, k)
    w8[0] = _int8(torch, 2, n, k)
    dw = _scales(torch, 3, experts, n)
    for rows in (3, 150):
        say("weights past 4 GiB", rows)
        x8, dx = _int8(torch, 4, rows, k), _scales(torch, 5, rows)
        chosen = torch.tensor([experts - 1, 0], dtype=torch.int32, device="cuda").repeat(rows)
        y = cq.cq_gemm_routed_w8(x8, dx, w8, dw, cq.cq_route_plan(chosen, experts), fan=2)
        for j, e in enumerate((experts - 1, 0)):
            assert torch.equal(y[j::2], cq.cq_gemm_w8(x8, dx, w8[e], dw[e]))
    del w8
    # rows of x and of y behind 4 GiB
    rows, n, k = 140000, 5, 32768
    say("activations past 4 GiB")
    x8 = torch.empty((rows, k), dtype=torch.int8, device="cuda")
    x8[-40:] = _int8(torch, 6, 40, k)
    dx, w8, dw = _scales(torch, 7, rows), _int8(torch, 8, n, k), _scales(torch, 9, n)
    y = cq.cq_gemm_w8(x8, dx, w8, dw, y_dtype=torch.float32)
    assert torch.equal(y[-40:], cq.cq_gemm_w8(x8[-40:], dx[-40:].clone(), w8, dw, y_dtype=torch.float32))
    chosen = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    chosen[-40:] = 0
    out = torch.zeros((rows, n), device="cuda")
    cq.cq_gemm_routed_w8(x8, dx, w8[None], dw[None], cq.cq_route_plan(chosen, 1), out=out)
    assert torch.equal(out[-40:], y[-40:]) and not bool(out[:-40].any())
    del x8
    rows, n, k = 70000, 65536, 16
    say("outputs past 4 GiB")
    x8, w8 = _int8(torch, 10, rows, k), _int8(torch, 11, n, k)
    dx, dw = _scales(torch, 12, rows), _scales(torch, 13, n)
    y = cq.cq_gemm_w8(x8, dx, w8, dw)
    assert torch.equal(y[-9:], cq.cq_gemm_w8(x8[-9:].clone(), dx[-9:].clone(), w8, dw))


# ---------------------------------------------------------------- gated activation


def _gated_ref(g, u, act):
    with np.errstate(over="ignore"):
        z = g if act == "silu" else np.sqrt(8.0 / np.pi) * (g + 0.044715 * g**3)
        return g / (1.0 + np.exp(-z)) * u, np.abs(z)


def _gated_bound(ref, z, dtype):
    # an exponent of z loses a few E z, what is left a few E
    return U[dtype] * np.abs(ref) + E * (16.0 + 8.0 * np.minimum(z, 128.0)) * np.abs(ref) + TINY


@pytest.mark.parametrize("rows,width", [(1, 8), (3, 504), (8, 2048), (2, 4104), (700, 1408), (5, 8192), (130, 14336),
                                        (1, 65536), (3000, 64)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gated(torch_dev, rows, width, act, dtype):
    torch, cq = torch_dev, _cq()
    fused = _rand(torch, 1, rows, 2 * width, dtype=dtype, scale=4.0)
    pairs = [fused.split(width, 1), fused.split(width, 1)[::-1],
             (_rand(torch, 2, rows, width, dtype=dtype, scale=9.0), _rand(torch, 3, rows, width, dtype=dtype)),
             _rand(torch, 4, rows, 2 * width + 24, dtype=dtype)[:, 8:8 + 2 * width].split(width, 1)]
    for n, (gate, up) in enumerate(pairs):
        say("gated", rows, width, act, dtype, n)
        ref, z = _gated_ref(_f64(gate), _f64(up), act)
        room = torch.full((rows * width + 64,), 7.0, dtype=_dtype(torch, dtype), device="cuda")
        got = cq.cq_gated(gate, up, act=act, out=room[:rows * width].view(rows, width))
        _within(got, ref, _gated_bound(ref, z, dtype), (act, n))
        assert bool((room[rows * width:] == 7.0).all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gated_of_every_value(torch_dev, act, dtype):
    torch, cq = torch_dev, _cq()
    gate = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(_dtype(torch, dtype)).cuda().view(8, 8192)
    up = torch.full_like(gate, -0.75)
    got = cq.cq_gated(gate, up, act=act)
    g = _f64(gate)
    fine = np.isfinite(g)
    with np.errstate(invalid="ignore"):
        ref, z = _gated_ref(np.where(fine, g, 0.0), -0.75, act)
    top = float(torch.finfo(_dtype(torch, dtype)).max)
    ok = fine & (np.abs(ref) < top)
    got = _f64(got)
    assert (np.abs(got - ref)[ok] <= _gated_bound(ref, z, dtype)[ok]).all()
    # NaN stays, +infinity goes through, -infinity has no value
    assert np.isnan(got[np.isnan(g)]).all() and np.isnan(got[g == -np.inf]).all() and (got[g == np.inf] == -np.inf).all()


@pytest.mark.parametrize("rows,width", [(1, 32), (8, 512), (5, 1024), (3, 2048), (600, 4096), (7, 4096), (9, 8192), (600, 8192),
                                        (4, 14336), (2, 32768), (3, 65536)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gated_to_carriers_equals_the_two_calls(torch_dev, rows, width, dtype):
    torch, cq = torch_dev, _cq()
    for act in ("silu", "gelu"):
        say("gated a8", rows, width, dtype, act)
        fused = _rand(torch, 5, rows, 2 * width, dtype=dtype, scale=3.0)
        if rows > 2:
            fused[1] = 0.0
        gate, up = fused.split(width, 1)
        h = torch.empty((rows, width), dtype=_dtype(torch, dtype), device="cuda")
        x8, dx = cq.cq_gated_a8(gate, up, act=act, out=h)
        assert torch.equal(h, cq.cq_gated(gate, up, act=act))
        want8, wantx = cq.cq_quantize_act_a8(h)
        assert torch.equal(x8, want8) and torch.equal(dx, wantx)
        again8, againx = cq.cq_gated_a8(gate, up, act=act)
        assert torch.equal(again8, want8) and torch.equal(againx, wantx)


def test_gated_of_more_elements_than_32_bits(torch_dev):
    torch, cq = torch_dev, _cq()
    rows, width = 70000, 65536
    gate = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    gate[-5:] = _rand(torch, 6, 5, width, dtype="bf16")
    out = cq.cq_gated(gate, gate)
    assert torch.equal(out[-5:], cq.cq_gated(gate[-5:], gate[-5:])) and not bool(out[:-5].any())


# ---------------------------------------------------------------- the experts joined


@pytest.mark.parametrize("tokens,top,width", [(1, 1, 8), (1, 8, 4096), (3, 5, 504), (130, 6, 4104), (700, 4, 1024), (2, 32, 256),
                                              (17, 3, 65536), (2500, 2, 64), (9, 12, 2048)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_combine(torch_dev, tokens, top, width, dtype):
    torch, cq = torch_dev, _cq()
    g = torch.Generator().manual_seed(tokens)
    for n, (base, alpha) in enumerate([(None, 1.0), ("same", 1.0), ("fp32", -0.5), ("same inplace", 2.0), (None, 0.25)]):
        say("combine", tokens, top, width, dtype, base, alpha)
        y = _rand(torch, 70 + n, tokens * top, width, dtype=dtype)
        weights = torch.rand((tokens, top), generator=g).cuda()
        chosen = torch.randint(-1, 9, (tokens, top), generator=g).to(torch.int32)
        if n == 1:
            chosen[0] = -1  # a token without experts
        lost = (chosen < 0) | (chosen >= 8)
        y[lost.flatten().cuda()] = float("nan")
        b = None
        if base:
            b = _rand(torch, 80 + n, tokens, width, dtype="fp32" if base == "fp32" else dtype)
        w = np.where(lost.numpy(), 0.0, _f64(weights))
        parts = np.nan_to_num(_f64(y)).reshape(tokens, top, width) * w[..., None] * alpha
        ref, mag = parts.sum(1), np.abs(parts).sum(1)
        if b is not None:
            ref, mag = ref + _f64(b), mag + np.abs(_f64(b))
        got = cq.cq_combine(y, weights, chosen.cuda(), 8, base=b, alpha=alpha, out=b if base == "same inplace" else None)
        if base == "same inplace":
            assert got is b
        u = U["fp32"] if base == "fp32" else U[dtype]
        _within(got, ref, u * np.abs(ref) + (top + 3) * E * mag + TINY, (n, base))
    wide = cq.cq_combine(y, weights, chosen.cuda(), 8, alpha=0.25, out=torch.empty((tokens, width), device="cuda"))
    _within(wide, ref, (top + 4) * E * mag, "fp32 out")


def test_combine_of_more_elements_than_32_bits(torch_dev):
    torch, cq = torch_dev, _cq()
    tokens, top, width = 40000, 2, 65536
    y = torch.zeros((tokens * top, width), dtype=torch.bfloat16, device="cuda")
    y[-6:] = _rand(torch, 7, 6, width, dtype="bf16")
    weights = torch.full((tokens, top), 0.5, device="cuda")
    chosen = torch.zeros((tokens, top), dtype=torch.int32, device="cuda")
    out = cq.cq_combine(y, weights, chosen, 1)
    assert torch.equal(out[-3:], cq.cq_combine(y[-6:], weights[-3:], chosen[-3:], 1)) and not bool(out[:-3].any())


# ---------------------------------------------------------------- together: a layer


def _layer(cq, s, stream=None):
    """Router to the joined experts, as a program runs it."""
    chosen, weights, plan = cq.cq_route(s["logits"], s["top"], scoring="sigmoid", bias=s["bias"], groups=4, kept_groups=2,
                                        group_top=2, scale=1.5, live=s["live"], stream=stream)
    x8, dx = cq.cq_quantize_act_a8(s["x"], stream=stream)
    pair = cq.cq_gemm_routed_w8(x8, dx, s["up"], s["dup"], plan, fan=s["top"], stream=stream)
    half = pair.shape[1] // 2
    h8, dh = cq.cq_gated_a8(pair[:, :half], pair[:, half:], stream=stream)
    y = cq.cq_gemm_routed_w8(h8, dh, s["down"], s["ddown"], plan, stream=stream)
    shared = cq.cq_gemm_w8(x8, dx, s["shared"], s["dshared"], stream=stream)
    return chosen, weights, plan, cq.cq_combine(y, weights, chosen, s["up"].shape[0], base=shared, stream=stream)


def _layer_inputs(torch, tokens, seed, experts=16, top=4, width=256, half=96):
    x = _rand(torch, seed, tokens, width, dtype="bf16")
    return {"x": x, "logits": _rand(torch, seed + 1, tokens, experts, dtype="fp32"), "top": top,
            "bias": _rand(torch, 2, experts, dtype="fp32", scale=0.1),
            "live": torch.tensor([tokens - tokens // 8], dtype=torch.int32, device="cuda"),
            "up": _int8(torch, 3, experts, 2 * half, width), "dup": _scales(torch, 4, experts, 2 * half),
            "down": _int8(torch, 5, experts, width, half), "ddown": _scales(torch, 6, experts, width),
            "shared": _int8(torch, 7, width, width), "dshared": _scales(torch, 8, width)}


def _layer_ref(torch, s, chosen, weights):
    """The layer from its chosen experts on, every operator from its definition; the
    roundings between two of them are part of the layer."""
    def carriers(v):
        d = np.maximum(np.abs(v).max(1), 1e-10) / 127.0
        return np.clip(np.floor(np.abs(v) / d[:, None] + 0.5), 0, 127) * np.sign(v), d

    def rounded(v):
        return _f64(torch.from_numpy(v).float().to(torch.bfloat16))

    x8, dx = carriers(_f64(s["x"]))
    out = rounded((x8 @ _f64(s["shared"]).T) * dx[:, None] * _f64(s["dshared"]))
    for t in range(len(chosen)):
        for j, e in enumerate(chosen[t]):
            if e < 0:
                continue
            pair = rounded(x8[t:t + 1] @ _f64(s["up"][e]).T * dx[t] * _f64(s["dup"][e]))
            half = pair.shape[1] // 2
            h = rounded(_gated_ref(pair[:, :half], pair[:, half:], "silu")[0])
            h8, dh = carriers(h)
            out[t] += weights[t, j] * rounded(h8 @ _f64(s["down"][e]).T * dh[:, None] * _f64(s["ddown"][e]))[0]
    return out


@pytest.mark.parametrize("tokens", [1, 9, 130])
def test_layer(torch_dev, tokens):
    torch, cq = torch_dev, _cq()
    s = _layer_inputs(torch, tokens, 10)
    chosen, weights, plan, out = _layer(cq, s)
    want, w = _route_ref(_f64(s["logits"]), 4, scoring="sigmoid", bias=_f64(s["bias"]), groups=4, kept_groups=2,
                         group_top=2, scale=1.5, live=int(s["live"].item()))
    assert np.array_equal(chosen.cpu().numpy(), want)
    ref = _layer_ref(torch, s, want, w)
    # one value in 2^8 of an intermediate may round to the other neighbour: 2^-8 of it, and
    # a carrier to the next one, 1 / 127 of the largest; in norm both stay below 2^-6
    off = np.linalg.norm(_f64(out) - ref, axis=1) / np.linalg.norm(ref, axis=1)
    assert off.max() < 2.0**-6


def test_layer_repeats_bit_for_bit_and_on_another_stream(torch_dev):
    torch, cq = torch_dev, _cq()
    s = _layer_inputs(torch, 300, 20)
    want = _layer(cq, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side, None, side):
        got = _layer(cq, s, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(want, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [1, 9, 500])
def test_layer_in_two_graphs(torch_dev, tokens):
    # replayed in turn, with new inputs and eager work between
    torch, cq = torch_dev, _cq()
    states = [_layer_inputs(torch, tokens, 30), _layer_inputs(torch, tokens, 40)]
    for s in states:
        _layer(cq, s)
    torch.cuda.synchronize()
    graphs = []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = _layer(cq, s)
        graphs.append((g, outs))
    for n in range(4):
        for s, (g, outs) in zip(states, graphs):
            fresh = _layer_inputs(torch, tokens, 50 + n)
            for name in ("x", "logits"):
                s[name].copy_(fresh[name])
            s["live"].fill_(max(1, tokens - n))
            g.replay()
            want = _layer(cq, s)
            torch.cuda.synchronize()
            for a, b in zip(want, outs):
                assert torch.equal(a, b)


def test_decoder_block_example_with_experts(torch_dev):
    from examples.decoder_block import serve
    errors = serve(experts=8, top=3, tokens=2, ffn=512, samples=3)
    # carriers are off by up to half a step, 1 / 254 of a row's largest value, which for
    # products of two normal values is up to some fifteen times their root mean square
    assert len(errors) == 2 * 5 and max(errors) < 15.0 / 254.0 + 2.0**-7


@pytest.mark.parametrize("experts,routes,n,k", [(5, 20, 40, 64), (70, 300, 40, 64), (5, 300, 40, 64), (16, 1000, 300, 144),
                                                (8, 4000, 400, 144), (48, 16000, 300, 1040), (8, 32000, 300, 1040)])
def test_offsets_far_from_each_other_lead_nowhere(torch_dev, experts, routes, n, k):
    # neighbours of a plan whose difference passes 32 bits, by kernels with tiles of 16 to
    # 256 rows: the routes of the runs that lie in the plan are written, and nothing else
    torch, cq = torch_dev, _cq()
    x8, dx = _int8(torch, 1, routes // 2, k), _scales(torch, 2, routes // 2)
    w8, dw = _int8(torch, 3, experts, n, k), _scales(torch, 4, experts, n)
    room = torch.full((routes + 40, n), 77.0, dtype=torch.bfloat16, device="cuda")
    most, order = 2**31 - 1, list(range(routes))
    for high, low in ((routes, -most), (most, -5), (most, -most - 1), (most, -most + routes // 2), (routes // 2 + 1, -most)):
        for rest, runs in (([low] * (experts - 1), ()), ([3] + [9] * (experts - 2), ((0, 3, 1), (3, 9, 2)))):
            say("offsets", experts, routes, n, k, high, low, len(runs))
            plan = torch.tensor([high, low] + rest + order, dtype=torch.int32, device="cuda")
            want = room.fill_(77.0).clone()
            for first, end, e in runs:
                r = torch.arange(first, end, device="cuda") // 2
                want[20 + first:20 + end] = cq.cq_gemm_w8(x8[r], dx[r], w8[e], dw[e])
            cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=2, out=room[20:20 + routes])
            torch.cuda.synchronize()
            assert torch.equal(room, want)


@pytest.mark.parametrize("n,k", [(700, 272), (6144, 400), (4099, 2064)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_product_with_a_bias_does_not_depend_on_the_kernel(torch_dev, n, k, dtype):
    # a row has the same bits whichever rows come with it, dense or routed
    torch, cq = torch_dev, _cq()
    x8, dx = _int8(torch, 1, 2500, k), _scales(torch, 2, 2500)
    w8, dw = _int8(torch, 3, 3, n, k), _scales(torch, 4, 3, n)
    bias, out = _rand(torch, 5, 3, n, dtype=dtype, scale=3.0), dict(y_dtype=_dtype(torch, dtype))
    one, done, bone = w8[1].clone(), dw[1].clone(), bias[1].clone()
    want = cq.cq_gemm_w8(x8, dx, one, done, bias=bone, **out)
    for rows in (1, 7, 9, 16, 17, 45, 100, 300, 700, 1300):
        say("bias", n, k, dtype, rows)
        got = cq.cq_gemm_w8(x8[:rows], dx[:rows], one, done, bias=bone, **out)
        assert torch.equal(got, want[:rows]), rows
        plan = cq.cq_route_plan(torch.ones((rows,), dtype=torch.int32, device="cuda"), 3)
        assert torch.equal(cq.cq_gemm_routed_w8(x8[:rows], dx[:rows], w8, dw, plan, bias=bias, **out), got), rows


@pytest.mark.parametrize("experts,groups", [(64, 8), (40, 5), (256, 16), (240, 3), (96, 32)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_of_groups_masked_by_the_lowest_bias(torch_dev, experts, groups, scoring):
    # a bias of FP32's lowest value is a choice like others: behind all that are not masked,
    # but in the group's sum of two beyond FP32
    torch = torch_dev
    size, low = experts // groups, torch.finfo(torch.float32).min
    for n, masked in enumerate([range(groups), range(1, groups), range(0, groups - 1), range(0, groups, 2)]):
        bias = _rand(torch, 90 + n, experts, dtype="fp32", scale=0.1)
        for g in masked:
            bias[g * size:(g + 1) * size] = low
        if n == 3:  # one that is not masked in a masked group
            bias[size // 2] = 0.25
        logits = _rand(torch, 95 + n, 33, experts, dtype="fp32", scale=2.0)
        for kept, top in ((1, 3), (2, 12), (min(groups - 1, 3), 4), (2, 16)):
            for group_top in (1, 2):
                say("masked groups", experts, groups, scoring, n, kept, top, group_top)
                _check_route(torch, logits, top, (n, kept, top, group_top), scoring=scoring, bias=bias, groups=groups,
                             kept_groups=kept, group_top=group_top)


@pytest.mark.parametrize("experts,groups,top", [(64, 8, 8), (256, 16, 12), (240, 3, 5), (96, 1, 8), (512, 4, 16), (600, 50, 7)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_of_the_largest_biases(torch_dev, experts, groups, top, scoring):
    # so large that scores vanish beside them, in FP64 too, and sums pass FP32
    torch = torch_dev
    most, inf = torch.finfo(torch.float32).max, float("inf")
    kinds = torch.tensor([most, -most, 2e38, -2e38, 1e30, -1e30, 0.0, 0.5, inf, -inf, float("nan"), -0.0])
    for seed in range(12):
        g = torch.Generator().manual_seed(seed)
        some = kinds[torch.randperm(len(kinds), generator=g)[:2 + seed % 4]]
        bias = some[torch.randint(0, len(some), (experts,), generator=g)].cuda()
        logits = _rand(torch, seed, 19, experts, dtype="fp32", scale=2.0)
        for kept, group_top in ((1, 1), (1, 2), (2, 2)):
            say("largest biases", experts, groups, top, scoring, seed, kept, group_top)
            _check_route(torch, logits, top, (seed, some), scoring=scoring, bias=bias, groups=groups,
                         kept_groups=min(kept, groups), group_top=group_top)


@pytest.mark.parametrize("low,high", [(-150.0, -89.0), (-115.0, -60.0), (-40.0, -5.0), (-700.0, -650.0), (-17.0, -15.0)])
@pytest.mark.parametrize("experts,top,groups", [(40, 6, 1), (256, 8, 8), (100, 20, 1), (64, 4, 32)])
def test_route_of_sigmoids_that_all_vanish(torch_dev, low, high, experts, top, groups):
    # scores below FP32's range have a sum to be divided by all the same
    torch = torch_dev
    g = torch.Generator().manual_seed(experts)
    logits = (low + (high - low) * torch.rand((37, experts), generator=g)).cuda()
    bias = _rand(torch, 9, experts, dtype="fp32", scale=0.1)
    for b in (None, bias):
        say("vanishing", low, high, experts, top, b is not None)
        _, weights, _ = _check_route(torch, logits, top, (low, b is None), scoring="sigmoid", bias=b, groups=groups,
                                     kept_groups=max(1, groups // 2))
        # each quotient and the sum of all are rounded
        assert bool(((weights.double().sum(1) - 1.0).abs() < (top + 8) * E).all())
    logits[::3, ::2] = -10.0  # beside scores that have not vanished
    _check_route(torch, logits, top, "beside", scoring="sigmoid", bias=bias, groups=groups, kept_groups=max(1, groups // 2))
    logits[5] = -2000.0  # FP64 has no such score
    assert not bool(_cq().cq_route(logits, top, scoring="sigmoid")[1][5].any())


@pytest.mark.parametrize("rows,n,k,kernel", W8_DENSE)
def test_product_by_every_kernel(torch_dev, rows, n, k, kernel):
    torch, cq = torch_dev, _cq()
    assert cq.cq_probe_w8_kernel(rows, n, k) == kernel
    x8, w8 = _int8(torch, rows + k, rows, k), _int8(torch, n + k, n, k)
    dx, dw = _scales(torch, 1, rows), _scales(torch, 2, n)
    for dtype in ("bf16", "fp16", "fp32"):
        for biased in (False, True):
            say("product by", kernel, rows, n, k, dtype, biased)
            bias = _rand(torch, 3, n, dtype=dtype) if biased else None
            # what lies before and behind the output stays
            room = torch.full((rows * n + 128,), 7.0, dtype=_dtype(torch, dtype), device="cuda")
            got = cq.cq_gemm_w8(x8, dx, w8, dw, bias=bias, out=room[64:64 + rows * n].view(rows, n))
            _check_on_device(torch, got, x8, dx, w8, dw, bias, dtype, (kernel, dtype, biased))
            assert bool((room[:64] == 7.0).all()) and bool((room[64 + rows * n:] == 7.0).all())


@pytest.mark.parametrize("experts,tokens,top,n,k,kernel", W8_ROUTED)
@pytest.mark.parametrize("fan", [True, False])
def test_routed_product_by_every_kernel(torch_dev, experts, tokens, top, n, k, kernel, fan):
    torch, cq = torch_dev, _cq()
    g = torch.Generator().manual_seed(experts * tokens)
    rows, per = (tokens, top) if fan else (tokens * top, 1)
    assert cq.cq_probe_w8_kernel(rows, n, k, experts, tokens * top, per) == kernel
    w8, dw = _int8(torch, 1, experts, n, k), _scales(torch, 2, experts, n)
    x8, dx = _int8(torch, 3, rows, k), _scales(torch, 4, rows)
    # some experts far more in demand than others, some routes of none
    chosen = (torch.rand((tokens, top), generator=g) ** 2 * (experts + 0.3)).long() - (torch.rand((tokens, top), generator=g) < 0.1).long()
    flat = chosen.flatten().cuda()
    plan = cq.cq_route_plan(chosen.to(torch.int32).cuda(), experts)
    for dtype, biased in (("bf16", True), ("fp16", False), ("fp32", True)):
        say("routed product by", kernel, experts, tokens, top, n, k, fan, dtype)
        bias = _rand(torch, 5, experts, n, dtype=dtype) if biased else None
        room = torch.full((tokens * top * n + 128,), 77.0, dtype=_dtype(torch, dtype), device="cuda")
        out = room[64:-64].view(tokens * top, n)
        cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=per, bias=bias, out=out)
        assert bool((out[(flat < 0) | (flat >= experts)] == 77.0).all())
        assert bool((room[:64] == 77.0).all()) and bool((room[-64:] == 77.0).all())
        for e in range(experts):
            r = (flat == e).nonzero()[:, 0]
            at = r // per
            if r.numel():
                _check_on_device(torch, out[r], x8[at], dx[at], w8[e], dw[e], None if bias is None else bias[e], dtype, e)


@pytest.mark.parametrize("rows,fan,dtype", [(65600, 2, "bf16"), (140000, 3, "fp16"), (131200, 1, "fp32")])
def test_routed_product_of_rows_behind_2_gib(torch_dev, rows, fan, dtype):
    # several experts, tiles that are full and not, a last step of 16 codes, rows of x up to
    # the last and behind 4 GiB: the same bits as the dense product of the same rows
    torch, cq = torch_dev, _cq()
    experts, n, k = 5, 203, 32784
    routes = rows * fan
    assert cq.cq_probe_w8_kernel(rows, n, k, experts, routes, fan) == ("tiles far", 128, 128, 2)
    say("far rows", rows, fan, dtype)
    g = torch.Generator().manual_seed(fan)
    x8 = torch.empty((rows, k), dtype=torch.int8, device="cuda")
    x8[:100], x8[-400:] = _int8(torch, 1, 100, k), _int8(torch, 2, 400, k)
    dx, w8, dw = _scales(torch, 3, rows), _int8(torch, 4, experts, n, k), _scales(torch, 5, experts, n)
    bias = _rand(torch, 6, experts, n, dtype=dtype)
    chosen = torch.full((rows, fan), -1, dtype=torch.int32)
    # the second expert has none, the fourth five
    share = torch.tensor([0, 0, 0, 2, 4], dtype=torch.int32)
    chosen[-400:] = share[torch.randint(0, 5, (400, fan), generator=g)]
    chosen[:100] = share[torch.randint(0, 5, (100, fan), generator=g)]
    chosen[-5:, 0] = 3
    flat = chosen.flatten().cuda()
    plan = cq.cq_route_plan(flat, experts)
    out = torch.full((routes, n), 77.0, dtype=_dtype(torch, dtype), device="cuda")
    cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=fan, bias=bias, out=out)
    assert bool((out[flat < 0] == 77.0).all())
    for e in range(experts):
        r = (flat == e).nonzero()[:, 0]
        if r.numel():
            x, d = x8[r // fan], dx[r // fan]
            want = cq.cq_gemm_w8(x, d, w8[e].clone(), dw[e].clone(), bias=bias[e].clone(), y_dtype=_dtype(torch, dtype))
            assert torch.equal(out[r], want), e
            _check_on_device(torch, out[r], x, d, w8[e], dw[e], bias[e], dtype, e)
    # offsets that are none
    # offsets far from each other, between which the third expert has all
    plan[:experts + 1] = torch.tensor([2**31 - 1, -5, -2**31 + 7, routes, -2**31 + 1, 0], dtype=torch.int32)
    out.fill_(77.0)
    x8.fill_(0)
    cq.cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=fan, out=out)
    assert bool((out[flat < 0] == 77.0).all()) and not bool(out[flat >= 0].any())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype,ups", [("bf16", (-0.75, 3.0, 2.0**60, -2.0**100)), ("fp16", (-0.75, 3.0, 1000.0))])
def test_gated_of_every_value_down_to_the_smallest(torch_dev, act, dtype, ups):
    # beside the half step of the output and the exponent's error, at most 2^-119 of up is
    # lost, where e^-v leaves FP32; FP16 has no such value
    torch, cq = torch_dev, _cq()
    gate = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(_dtype(torch, dtype)).cuda().view(8, 8192)
    g, most = _f64(gate), float(torch.finfo(_dtype(torch, dtype)).max)
    half_step = {"bf16": 2.0**-134, "fp16": 2.0**-25}[dtype]
    for u in ups:
        say("gated, small", act, dtype, u)
        got = _f64(cq.cq_gated(gate, torch.full_like(gate, u), act=act))
        with np.errstate(invalid="ignore"):
            ref, z = _gated_ref(np.where(np.isfinite(g), g, 0.0), u, act)
        ok = np.isfinite(g) & (np.abs(ref) < most)
        bound = U[dtype] * np.abs(ref) + E * (16.0 + 8.0 * np.minimum(z, 128.0)) * np.abs(ref) + half_step + 2.0**-119 * abs(u)
        off = np.where(ok, np.abs(got - ref) - bound, -1.0)
        assert (off <= 0).all(), (u, g.ravel()[np.argmax(off)])


@pytest.mark.parametrize("tokens,experts,top", [(1, 128, 8), (31, 64, 6), (700, 256, 8), (5, 1000, 32), (90, 72, 16)])
@pytest.mark.parametrize("biased", [False, True])
def test_route_without_a_plan(torch_dev, tokens, experts, top, biased):
    # from C, which leaves the plan and its workspace out
    torch, cq = torch_dev, _cq()
    from paper_2608_06763_amd import experts as X
    say("no plan", tokens, experts, top, biased)
    logits = _rand(torch, 1, tokens, experts, dtype="fp32", scale=2.0)
    bias = _rand(torch, 2, experts, dtype="fp32", scale=0.1) if biased else None
    live = torch.tensor([tokens - tokens // 4], dtype=torch.int32, device="cuda")
    want = cq.cq_route(logits, top, bias=bias, live=live)
    chosen = torch.full((tokens * top + 8,), -77, dtype=torch.int32, device="cuda")
    weights = torch.full((tokens * top + 8,), 77.0, device="cuda")
    args = X._ROUTE.pack(logits.data_ptr(), bias.data_ptr() if biased else 0, live.data_ptr(), chosen.data_ptr(),
                         weights.data_ptr(), 0, tokens, experts, 2, experts, top, 0, 1, 1, 1, 1, 1.0)
    assert cq.lib().cq_route_workspace_bytes(args) == 0
    assert cq.lib().cq_route(args, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(chosen[:-8].view(tokens, top), want[0]) and torch.equal(weights[:-8].view(tokens, top), want[1])
    assert bool((chosen[-8:] == -77).all()) and bool((weights[-8:] == 77.0).all())


@pytest.mark.parametrize("tokens,experts,top", [(70001, 256, 8), (40000, 100, 1), (16385, 1024, 6), (16384, 64, 16), (131072, 12, 3),
                                                (20000, 60, 20)])
def test_route_of_many_tokens_equals_its_parts(torch_dev, tokens, experts, top):
    torch, cq = torch_dev, _cq()
    g = torch.Generator(device="cuda").manual_seed(tokens)
    logits = torch.randn((tokens, experts), generator=g, device="cuda").to(torch.bfloat16)
    bias = _rand(torch, 2, experts, dtype="fp32", scale=0.1)
    live = torch.tensor([tokens - 77], dtype=torch.int32, device="cuda")
    for kw in (dict(bias=bias, scoring="sigmoid"), dict(), dict(bias=bias, groups=4, kept_groups=2, group_top=2)):
        if kw.get("groups") and top > experts // 2:
            continue
        say("many tokens", tokens, experts, top, sorted(kw))
        chosen, weights, plan = cq.cq_route(logits, top, live=live, **kw)
        for t in range(0, tokens, 3000):
            rest = torch.tensor([max(0, min(3000, tokens - 77 - t))], dtype=torch.int32, device="cuda")
            part = cq.cq_route(logits[t:t + 3000], top, live=rest, **kw)
            assert torch.equal(chosen[t:t + 3000], part[0]) and torch.equal(weights[t:t + 3000], part[1]), t
        assert np.array_equal(plan.cpu().numpy(), _plan_ref(chosen.cpu().numpy(), experts))


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_route_of_infinities_by_every_search(torch_dev, scoring, dtype):
    # the exact search alone (more than twelve choices) and a wave a token (more than sixteen
    # choices, or groups)
    torch = torch_dev
    inf, nan = float("inf"), float("nan")
    low, most = torch.finfo(_dtype(torch, dtype)).min, torch.finfo(_dtype(torch, dtype)).max
    logits = _rand(torch, 44, 13, 96, dtype=dtype)
    logits[0], logits[1] = -inf, nan
    logits[2, ::2], logits[3, 1::3] = -inf, nan
    logits[4, 5], logits[4, 50] = inf, inf
    logits[5] = low
    logits[6] = -inf
    logits[6, 95] = 1.0
    logits[7, :94] = nan
    logits[8, 3:] = low
    logits[9] = inf
    logits[10, 10:] = -60.0
    logits[11, ::7] = most
    bias = _rand(torch, 45, 96, dtype="fp32", scale=0.1)
    odd = bias.clone()
    odd[:40], odd[40], odd[41], odd[50:70] = -inf, nan, inf, torch.finfo(torch.float32).min
    for n, (top, opt) in enumerate([(14, dict(bias=bias)), (16, dict(bias=odd)), (15, dict()), (20, dict()), (20, dict(bias=odd)),
                                    (32, dict(renormalize=False)), (6, dict(groups=32, kept_groups=5, group_top=2)),
                                    (6, dict(groups=32, kept_groups=9, group_top=2, bias=odd)),
                                    (14, dict(groups=12, kept_groups=4, group_top=2, bias=odd)),
                                    (6, dict(groups=48, kept_groups=3, bias=bias)), (6, dict(groups=48, kept_groups=3))]):
        say("route odd values, searches", scoring, dtype, n)
        _check_route(torch, logits, top, n, scoring=scoring, **opt)


@pytest.mark.parametrize("width", [64, 1024, 4096, 14336])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gated_to_carriers_of_odd_values(torch_dev, width, dtype):
    torch, cq = torch_dev, _cq()
    gate, up = _rand(torch, 1, 9, width, dtype=dtype, scale=3.0), _rand(torch, 2, 9, width, dtype=dtype)
    inf, info = float("inf"), torch.finfo(_dtype(torch, dtype))
    gate[0, 3], gate[1, 5], gate[2] = inf, float("nan"), -inf
    up[3, 7], up[4, ::9], gate[5] = -inf, float("nan"), 0.0
    gate[6], up[6] = info.max, info.max
    gate[7], up[7] = info.tiny, info.tiny
    up[8, :-1] = info.smallest_normal
    for act in ("silu", "gelu"):
        say("gated a8, odd values", width, dtype, act)
        h = torch.empty_like(gate)
        x8, dx = cq.cq_gated_a8(gate, up, act=act, out=h)
        assert torch.equal(h.view(torch.int16), cq.cq_gated(gate, up, act=act).view(torch.int16))
        want8, wantx = cq.cq_quantize_act_a8(h)
        assert torch.equal(x8, want8) and torch.equal(dx.view(torch.int32), wantx.view(torch.int32))


def test_combine_of_odd_values(torch_dev):
    # routes without an expert give nothing, whatever their weights and rows hold; others
    # what the sum gives
    torch, cq = torch_dev, _cq()
    inf, nan = float("inf"), float("nan")
    y = torch.ones((5 * 3, 16), dtype=torch.bfloat16, device="cuda")
    chosen = torch.tensor([[-1, 7, 2**31 - 1], [0, -2**31, 1], [2, 2, 2], [3, 0, 1], [-1, -1, -1]], dtype=torch.int32, device="cuda")
    weights = torch.tensor([[nan, inf, -inf], [0.5, nan, 0.25], [1.0, 2.0, 4.0], [inf, 1.0, 1.0], [nan] * 3], device="cuda")
    y[:3], y[4] = nan, inf
    got = cq.cq_combine(y, weights, chosen, 4, out=torch.empty((5, 16), device="cuda"))
    assert torch.equal(got, torch.tensor([0.0, 0.75, 7.0, inf, 0.0], device="cuda")[:, None].expand(5, 16))
