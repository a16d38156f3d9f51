"""GPU: the operators between the packed products against plain 64-bit forms.

Tolerances.  u is the unit roundoff of the output's type (2^-8 BF16, 2^-11
FP16): the one rounding of an output costs u |y|.  FP32 sums of up to a few ten
thousand terms and the hardware's exp and rsqrt stay within 2^-15 relative; a
score of magnitude s adds s 2^-22 to the weight, below 2^-15 for the scores here.
Attention may round its weights to the cache's type, u of sum(p |v|) more.
"""
import numpy as np
import pytest

from tests._cases import say

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0**-8, "fp16": 2.0**-11}
FP32 = 2.0**-15
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
    return torch.bfloat16 if name == "bf16" else torch.float16


def _rand(torch, seed, *shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(_dtype(torch, dtype)).cuda()


def _f64(t):
    return t.detach().cpu().double().numpy()


def _within(got, ref, bound, what):
    got = _f64(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), what
    off = np.abs(got - ref) - bound
    assert (off <= 0).all(), f"{what}: {np.max(off)} over the bound at {np.unravel_index(np.argmax(off), off.shape)}"


# ---------------------------------------------------------------- norms


def _norm_ref(r, w, eps, off, y, wp, gate, alpha):
    if y is None:
        total, mag = r, np.abs(r)
    else:
        u = y
        if wp is not None:
            u = u / np.sqrt((u * u).mean(1, keepdims=True) + eps) * (wp + off)
        if gate is not None:
            u = u * gate
        total, mag = r + alpha * u, np.abs(r) + np.abs(alpha * u)
    h = total / np.sqrt((total * total).mean(1, keepdims=True) + eps) * (w + off)
    slack = mag / np.sqrt((total * total).mean(1, keepdims=True) + eps) * np.abs(w + off)
    return h, total, mag, slack


NORM_FORMS = [
    dict(), dict(y=True), dict(y=True, post=True, off=1.0), dict(y=True, gate="row", alpha=-0.25),
    dict(y=True, gate="all", post=True, r32=True), dict(y=True, r32=True, inplace=True, alpha=0.5),
    dict(y=True, gate="strided", post=True, inplace=True),
]


@pytest.mark.parametrize("rows,width", [(1, 8), (3, 504), (5, 1024), (2, 2040), (1, 4096), (130, 4104), (600, 2056),
                                        (2, 8192), (520, 8192), (3, 16384), (2, 32768)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_norm_residual(torch_dev, rows, width, dtype):
    torch, cq = torch_dev, _cq()
    for n, f in enumerate(NORM_FORMS):
        say("norm", rows, width, dtype, f)
        r = _rand(torch, 10 + n, rows, width, dtype=dtype, scale=3.0)
        if f.get("r32"):
            r = r.float() * 1.2345
        w = _rand(torch, 20 + n, width, dtype=dtype)
        y = _rand(torch, 30 + n, rows, width, dtype=dtype) if f.get("y") else None
        wp = _rand(torch, 40 + n, width, dtype=dtype) if f.get("post") else None
        gate = None
        if f.get("gate") == "row":
            gate = _rand(torch, 50 + n, rows, width, dtype=dtype)
        elif f.get("gate") == "strided":
            gate = _rand(torch, 50 + n, rows, width + 16, dtype=dtype)[:, 8:8 + width]
        elif f.get("gate"):
            gate = _rand(torch, 50 + n, width, dtype=dtype)
        alpha, off = f.get("alpha", 1.0), f.get("off", 0.0)
        opt = [None if t is None else _f64(t) for t in (y, wp, gate)]
        h_ref, r_ref, mag, slack = _norm_ref(_f64(r), _f64(w), 1e-5, off, *opt, alpha)
        h, r_out = cq.cq_norm_residual(r, w, 1e-5, y=y, post_weight=wp, gate=gate, alpha=alpha, weight_offset=off,
                                       out=y if f.get("inplace") else None,
                                       residual_out=r if f.get("inplace") else None)
        _within(h, h_ref, U[dtype] * np.abs(h_ref) + FP32 * slack + TINY, "h")
        ur = 2.0**-24 if f.get("r32") else U[dtype]
        if y is None:
            assert r_out is r
        else:
            _within(r_out, r_ref, ur * np.abs(r_ref) + FP32 * mag + TINY, "residual")


def test_norm_of_zero_rows_and_not_a_number(torch_dev):
    torch, cq = torch_dev, _cq()
    r = torch.zeros((4, 256), dtype=torch.bfloat16, device="cuda")
    r[1] = 3.0
    r[2, 7] = float("nan")
    w = torch.ones((256,), dtype=torch.bfloat16, device="cuda")
    h, _ = cq.cq_norm_residual(r, w, 1e-6)
    assert bool((h[0] == 0).all()) and bool((h[3] == 0).all()) and bool((h[1] == 1).all())
    assert bool(torch.isnan(h[2]).all())


@pytest.mark.parametrize("rows,width", [(1, 4096), (7, 96), (3, 1056), (70, 8192), (600, 2048), (600, 8192), (2, 14336)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_norm_to_carriers_equals_the_two_calls(torch_dev, rows, width, dtype):
    torch, cq = torch_dev, _cq()
    say("norm a8", rows, width, dtype)
    r, y = (_rand(torch, 60 + i, rows, width, dtype=dtype, scale=2.0) for i in range(2))
    w, wp = (_rand(torch, 70 + i, width, dtype=dtype) for i in range(2))
    h, r_out = cq.cq_norm_residual(r, w, 1e-5, y=y, post_weight=wp)
    x8_ref, dx_ref = cq.cq_quantize_act_a8(h)
    out = torch.empty_like(h)
    x8, dx, r8 = cq.cq_norm_residual_a8(r, w, 1e-5, y=y, post_weight=wp, out=out)
    assert torch.equal(x8, x8_ref) and torch.equal(dx, dx_ref) and torch.equal(out, h) and torch.equal(r8, r_out)
    x8, dx, _ = cq.cq_norm_residual_a8(r, w, 1e-5, y=y, post_weight=wp)
    assert torch.equal(x8, x8_ref) and torch.equal(dx, dx_ref)


@pytest.mark.parametrize("rows,width", [(1, 64), (5, 1056), (600, 8192)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("r32", [False, True])
@pytest.mark.parametrize("a8", [False, True])
def test_norm_without_y_writes_the_residual_too(torch_dev, rows, width, dtype, r32, a8):
    # r' = residual: into the buffer of its own that the caller names
    import ctypes
    torch, cq = torch_dev, _cq()
    say("norm without y", rows, width, dtype, r32, a8)
    r, w = _rand(torch, 11, rows, width, dtype=dtype, scale=2.0), _rand(torch, 12, width, dtype=dtype)
    r = r.float() * 1.2345 if r32 else r
    kind = {"bf16": cq.CQ_BF16, "fp16": cq.CQ_FP16}[dtype]
    h, r_out = torch.full_like(r, 7.0, dtype=w.dtype), torch.full_like(r, 7.0)
    args = cq.block.cq_norm_args(
        y=None, post_weight=None, gate=None, residual=r.data_ptr(), weight=w.data_ptr(), residual_out=r_out.data_ptr(),
        out=h.data_ptr(), gate_stride=0, rows=rows, width=width, dtype=kind,
        residual_dtype=cq.CQ_FP32 if r32 else kind, alpha=1.0, eps=1e-5, weight_offset=0.0)
    x8, dx = torch.empty((rows, width), dtype=torch.int8, device="cuda"), torch.empty((rows,), device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    if a8:
        assert cq.lib().cq_norm_residual_a8(ctypes.byref(args), x8.data_ptr(), dx.data_ptr(), stream) == 0
    else:
        assert cq.lib().cq_norm_residual(ctypes.byref(args), stream) == 0
    assert torch.equal(r_out, r)
    h_ref, _, _, slack = _norm_ref(_f64(r), _f64(w), 1e-5, 0.0, None, None, None, 1.0)
    _within(h, h_ref, U[dtype] * np.abs(h_ref) + FP32 * slack + TINY, "h")
    # and through the binding
    copy = torch.full_like(r, 7.0)
    if a8:
        _, _, same = cq.cq_norm_residual_a8(r, w, 1e-5, residual_out=copy)
    else:
        again, same = cq.cq_norm_residual(r, w, 1e-5, residual_out=copy)
        assert torch.equal(again, h)
    assert same is copy and torch.equal(copy, r)


# ---------------------------------------------------------------- rotation and append


def _turn(x, cos, sin, interleaved):
    """Rotated x and the sum of the magnitudes that make each channel."""
    rot = 2 * cos.shape[1]
    out, mag = x.copy(), np.abs(x)
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    c, s, a, b = cos[:, None], sin[:, None], x[..., lo], x[..., hi]
    out[..., lo], out[..., hi] = a * c - b * s, b * c + a * s
    mag[..., lo], mag[..., hi] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return out, mag


@pytest.mark.parametrize("dim,rot,interleaved", [(64, 64, False), (64, 16, False), (128, 128, False), (128, 96, True),
                                                 (256, 256, True), (256, 64, False), (128, 0, False)])
@pytest.mark.parametrize("tokens,heads,kv_heads,page,dtype", [(1, 4, 1, 16, "bf16"), (37, 6, 3, 32, "fp16"),
                                                              (300, 35, 5, 128, "bf16")])
def test_rope_append(torch_dev, dim, rot, interleaved, tokens, heads, kv_heads, page, dtype):
    torch, cq = torch_dev, _cq()
    say("append", dim, rot, interleaved, tokens, heads, kv_heads, page, dtype)
    g = torch.Generator().manual_seed(3)
    pages, rows = tokens // page + 3, 500
    qkv = _rand(torch, 80, tokens, heads + 2 * kv_heads, dim, dtype=dtype)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    angle = torch.randn((rows, rot // 2), generator=g).cuda()
    cos, sin = (angle.cos(), angle.sin()) if rot else (None, None)
    positions = torch.randint(0, rows, (tokens,), generator=g).to(torch.int32)
    slots = torch.randperm(pages * page, generator=g)[:tokens].to(torch.int32)
    if tokens > 2:
        slots[1], slots[2] = -1, pages * page  # not appended
    caches = [_rand(torch, 90 + i, pages, kv_heads, page, dim, dtype=dtype) for i in range(2)]
    before = [_f64(c) for c in caches]
    q_out = cq.cq_rope_append(q, k, v, cos, sin, positions.cuda(), slots.cuda(), *caches, interleaved=interleaved)
    at = positions.numpy()
    cn, sn = (_f64(cos)[at], _f64(sin)[at]) if rot else (np.zeros((tokens, 0)), np.zeros((tokens, 0)))
    for got, x in ((q_out, q), (None, k)):
        ref, mag = _turn(_f64(x), cn, sn, interleaved)
        bound = U[dtype] * np.abs(ref) + 2.0**-22 * mag + TINY
        if got is not None:
            _within(got, ref, bound, "q")
            continue
        k_ref, k_bound = before[0].copy(), np.zeros_like(before[0])
        v_ref = before[1].copy()
        for i, s in enumerate(slots.tolist()):
            if 0 <= s < pages * page:
                k_ref[s // page, :, s % page], k_bound[s // page, :, s % page] = ref[i], bound[i]
                v_ref[s // page, :, s % page] = _f64(v)[i]
        _within(caches[0], k_ref, k_bound, "k")  # untouched slots: exactly
        assert np.array_equal(_f64(caches[1]), v_ref)
    # in place, on the fused product
    same = cq.cq_rope_append(q, k, v, cos, sin, positions.cuda(), slots.cuda(), *caches, interleaved=interleaved,
                             q_out=q)
    assert same is q and torch.equal(q, q_out)


def test_rope_positions_outside_the_tables_are_clamped(torch_dev):
    torch, cq = torch_dev, _cq()
    q, kv = _rand(torch, 1, 3, 2, 64, dtype="bf16"), _rand(torch, 2, 3, 1, 64, dtype="bf16")
    angle = torch.arange(5 * 32, device="cuda").view(5, 32).float()
    slots = torch.arange(3, device="cuda", dtype=torch.int32)

    def go(p):
        caches = [torch.zeros((1, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        pos = torch.tensor(p, device="cuda", dtype=torch.int32)
        return cq.cq_rope_append(q, kv, kv, angle.cos(), angle.sin(), pos, slots, *caches)

    assert torch.equal(go([-7, 5, 1 << 30]), go([0, 4, 4]))


# ---------------------------------------------------------------- attention


def _paged(torch, seed, lens, page, kv_heads, dim, dtype, spare=3, garbage=float("nan")):
    """Caches whose pages lie in random order, with `garbage` wherever no token is
    held, and tables with wild entries past each sequence's end; and the keys and
    values of every sequence."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages, width = sum(need) + spare, max(max(need), 1) + 1
    order = torch.randperm(pages, generator=g)
    pools = [torch.full((pages, kv_heads, page, dim), garbage) for _ in range(2)]
    tables = torch.full((len(lens), width), -5, dtype=torch.int32)
    tables[:, -1] = 1 << 30
    held, at = [], 0
    for b, n in enumerate(lens):
        own = order[at:at + need[b]]
        at += need[b]
        tables[b, :need[b]] = own.to(torch.int32)
        kv = []
        for i, pool in enumerate(pools):
            x = torch.randn((n, kv_heads, dim), generator=g) + (0.2 if i else 0.0)
            x = x.to(_dtype(torch, dtype)).float()
            for p in range(need[b]):
                part = x[p * page:(p + 1) * page]
                pool[own[p], :, :part.shape[0]] = part.transpose(0, 1)
            kv.append(x.double().numpy())
        held.append(kv)
    return [p.to(_dtype(torch, dtype)).cuda() for p in pools], tables.cuda(), held


def _attn_ref(q, held, new, scale, softcap=0.0, window=0, slopes=None, bidir=None, prefix=None):
    """Outputs, and sum(p |v|), per row of q [tokens, heads, dim]."""
    tokens, heads, dim = q.shape
    out, mag, row = np.zeros_like(q), np.zeros_like(q), 0
    for b, n in enumerate(new):
        k, v = held[b]
        length, group = k.shape[0], heads // k.shape[1]
        i = np.arange(length - n, length)[:, None]
        j = np.arange(length)[None]
        seen = j <= i
        if window:
            seen &= j > i - window
        if bidir is not None:
            seen |= (j < bidir[b]) & (i >= 0)
        for h in range(heads):
            s = q[row:row + n, h] @ k[:, h // group].T * scale
            if softcap:
                s = softcap * np.tanh(s / softcap)
            if slopes is not None:
                s = s + slopes[h] * (j - i)
            s = np.where(seen, s, -np.inf)
            vv = v[:, h // group]
            if prefix is not None:
                f = q[row:row + n, h] @ prefix[0][:, h // group].T * scale
                if softcap:
                    f = softcap * np.tanh(f / softcap)
                s, vv = np.concatenate((f, s), 1), np.concatenate((prefix[1][:, h // group], vv))
            if n == 0 or s.shape[1] == 0:
                continue
            top = s.max(1, keepdims=True)
            p = np.exp(s - np.where(np.isinf(top), 0.0, top))
            p = p / np.where(p.sum(1, keepdims=True) > 0, p.sum(1, keepdims=True), 1.0)
            # hidden tokens do not reach the output, whatever they hold
            used = np.where(p.max(0) > 0, 1.0, 0.0)[:, None]
            vv = np.where(used > 0, vv, 0.0)
            out[row:row + n, h], mag[row:row + n, h] = p @ vv, p @ np.abs(vv)
        row += n
    return out, mag


def _check_attn(torch, dtype, dim, heads, kv_heads, page, new, lens, seed=5, max_kv=None, starts=None, garbage=np.nan,
                **opt):
    cq = _cq()
    say("attn", dtype, dim, heads, kv_heads, page, new, lens, {k: v for k, v in opt.items() if k != "slopes"})
    caches, tables, held = _paged(torch, seed, lens, page, kv_heads, dim, dtype, garbage=garbage)
    total = sum(new)
    qkv = _rand(torch, seed + 1, total, heads + 2 * kv_heads, dim, dtype=dtype, scale=1.5)
    q = qkv[:, :heads]
    if starts is None and max(new) > 1 or min(new) != 1:
        starts = torch.tensor(np.cumsum([0] + new), dtype=torch.int32).cuda()
    args = dict(opt)
    for name, kind in (("slopes", torch.float32), ("bidir", torch.int32)):
        if args.get(name) is not None:
            args[name] = torch.tensor(args[name], dtype=kind).cuda()
    out = cq.cq_attn_paged(q, *caches, tables, torch.tensor(lens, dtype=torch.int32).cuda(),
                           max(max(lens), 0) if max_kv is None else max_kv, q_starts=starts, max_q=max(new), **args)
    ref, mag = _attn_ref(_f64(q), held, new, opt.pop("scale", dim**-0.5), **opt)
    u = U[dtype]
    _within(out, ref, u * np.abs(ref) + (u + FP32) * mag + TINY, "attention")
    return out


# lengths on both sides of the edges of pages and of tiles of 16, 32, 64, 128
LENS = [1, 15, 16, 17, 31, 32, 33, 64, 65, 127, 129, 300]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2), (7, 1), (20, 4), (33, 1), (16, 16)])
@pytest.mark.parametrize("page", [16, 64])
def test_attn_single_tokens(torch_dev, dtype, dim, heads, kv_heads, page):
    _check_attn(torch_dev, dtype, dim, heads, kv_heads, page, [1] * len(LENS), LENS)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,page", [(2, 2, 16), (8, 2, 32), (5, 1, 128)])
@pytest.mark.parametrize("new,lens", [
    ([1, 2, 3, 7, 8, 4], [1, 2, 30, 64, 65, 400]),          # a few tokens each
    ([5, 33, 64, 17, 1], [5, 33, 64, 17, 1]),               # prompts
    ([130, 257, 63], [130, 300, 190]),                      # prompts and chunks
    ([0, 3, 0, 1, 0], [40, 3, 0, 9, 7]),                    # sequences without queries
])
def test_attn_ragged(torch_dev, dtype, dim, heads, kv_heads, page, new, lens):
    _check_attn(torch_dev, dtype, dim, heads, kv_heads, page, new, lens)


OPTIONS = [dict(softcap=5.0), dict(window=1), dict(window=20), dict(window=100), dict(scale=0.31),
           dict(slopes=[0.5, 0.01, 0.25, 1.0]), dict(softcap=8.0, window=50, slopes=[0.1, 0.3, 0.0, 2.0]),
           dict(bidir=[0, 7, 500, 33, 1]), dict(bidir=[90, 0, 64, 5, 1], window=16, softcap=20.0)]


@pytest.mark.parametrize("opt", OPTIONS, ids=str)
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("bf16", 256)])
@pytest.mark.parametrize("new,lens", [([1, 1, 1, 1, 1], [1, 40, 129, 33, 290]), ([4, 6, 2, 1, 5], [4, 70, 129, 40, 33]),
                                      ([90, 200, 64, 33, 140], [90, 230, 64, 300, 140])])
def test_attn_scores_and_masks(torch_dev, opt, dtype, dim, new, lens):
    _check_attn(torch_dev, dtype, dim, 4, 2, 16, new, lens, **opt)


@pytest.mark.parametrize("new,lens", [([1, 1, 1], [0, 1, 0]), ([3, 5, 2], [0, 2, 9]), ([100, 150], [20, 0]),
                                      ([1], [0])])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("fp16", 256)])
def test_attn_rows_that_see_nothing_are_zero(torch_dev, dtype, dim, new, lens):
    out = _check_attn(torch_dev, dtype, dim, 4, 2, 16, new, lens, bidir=[4] * len(new))
    row = 0
    for n, length in zip(new, lens):
        assert bool((out[row:row + max(0, n - length)] == 0).all())
        row += n


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new", [3, 40, 150])
def test_attn_hidden_tokens_may_hold_anything(torch_dev, dtype, dim, bad, new):
    # the last token's value (and key, if no number) is bad: all queries but the
    # last are as before, up to the rounding of outputs and weights on either side
    # (2 u of a mean magnitude below 2)
    torch, cq = torch_dev, _cq()
    say("attn hidden", dtype, dim, bad, new)
    heads, kv_heads, page, length = 4, 2, 16, new + 21
    caches, tables, held = _paged(torch, 9, [length], page, kv_heads, dim, dtype, garbage=bad)
    q = _rand(torch, 10, new, heads, dim, dtype=dtype)
    starts = torch.tensor([0, new], dtype=torch.int32).cuda()
    lens = torch.tensor([length], dtype=torch.int32).cuda()
    good = cq.cq_attn_paged(q, *caches, tables, lens, length, q_starts=starts, max_q=new)
    at = int(tables[0, (length - 1) // page])
    caches[1][at, :, (length - 1) % page] = bad
    if bad != bad:
        caches[0][at, 0, (length - 1) % page, 1] = bad
    out = cq.cq_attn_paged(q, *caches, tables, lens, length, q_starts=starts, max_q=new)
    near = dict(rtol=2 * U[dtype], atol=4 * U[dtype])
    assert torch.allclose(out[:-1].float(), good[:-1].float(), **near)
    assert not bool(torch.isfinite(out[-1]).any())
    # and one that the window has left behind
    caches[1][at, :, (length - 1) % page] = 1.0
    caches[0][at, 0, (length - 1) % page, 1] = 1.0
    base = cq.cq_attn_paged(q, *caches, tables, lens, length, q_starts=starts, max_q=new, window=5)
    caches[1][int(tables[0, 0]), :, 3] = bad
    caches[1][int(tables[0, 1]), :, 1] = bad  # token 17: the first query (21) just sees it
    out = cq.cq_attn_paged(q, *caches, tables, lens, length, q_starts=starts, max_q=new, window=5)
    assert torch.allclose(out[1:].float(), base[1:].float(), **near) and not bool(torch.isfinite(out[0]).any())


def test_attn_long_history(torch_dev):
    _check_attn(torch_dev, "bf16", 128, 8, 2, 64, [1], [5003])
    _check_attn(torch_dev, "fp16", 64, 4, 2, 16, [1, 2, 1], [4000, 9, 1700])
    _check_attn(torch_dev, "fp16", 64, 4, 1, 128, [70, 2], [4000, 3])


def test_attn_many_sequences(torch_dev):
    rng = np.random.default_rng(4)
    lens = [int(n) for n in rng.integers(0, 90, 700)]
    _check_attn(torch_dev, "bf16", 64, 2, 1, 16, [1] * 700, lens)


def test_attn_bounds_cut_the_sequences(torch_dev):
    # lengths past max_kv, or past the table, are cut; nothing outside is read
    torch, cq = torch_dev, _cq()
    caches, tables, held = _paged(torch, 2, [64, 40], 16, 1, 64, "bf16")
    q = _rand(torch, 3, 2, 2, 64, dtype="bf16")

    def go(lens, max_kv, table):
        return cq.cq_attn_paged(q, *caches, table.contiguous(), torch.tensor(lens, dtype=torch.int32).cuda(), max_kv)

    want = go([40, 40], 40, tables)
    assert torch.equal(go([2**31 - 1, 41], 40, tables), want)
    assert torch.equal(go([48, -3], 1000, tables)[0], go([1000, -3], 1000, tables[:, :3])[0])
    assert bool((go([48, -3], 1000, tables)[1] == 0).all())


def test_attn_large_scores(torch_dev):
    # one token far above the others, and equal scores of large magnitude
    torch, cq = torch_dev, _cq()
    for dtype in ("bf16", "fp16"):
        caches, tables, held = _paged(torch, 6, [150, 150], 16, 1, 64, dtype)
        for c, table in ((caches[0], tables),):
            c[int(table[0, 2]), 0, 5] = 30.0
            c[table[1, :10].long()] = -60.0
        held[0][0][37, 0] = 30.0
        held[1][0][:] = -60.0
        q = torch.full((2, 2, 64), 10.0, dtype=_dtype(torch, dtype), device="cuda")
        out = cq.cq_attn_paged(q, *caches, tables, torch.tensor([150, 150], dtype=torch.int32).cuda(), 150)
        ref, mag = _attn_ref(_f64(q), held, [1, 1], 0.125)
        _within(out, ref, U[dtype] * np.abs(ref) + (U[dtype] + FP32) * mag + TINY, "large scores")


def test_attn_offsets_past_32_bits(torch_dev):
    # pools of 6 GiB each; the sequence lies at their ends
    torch, cq = torch_dev, _cq()
    kv_heads, page, dim, length = 8, 64, 128, 700
    pages = (6 << 30) // (kv_heads * page * dim * 2)
    pools = [torch.empty((pages, kv_heads, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n = -(-length // page)
    own = torch.tensor([pages - 1 - 2 * i for i in range(n)])
    x = [_rand(torch, 11 + i, n, kv_heads, page, dim, dtype="bf16") for i in range(2)]
    for pool, part in zip(pools, x):
        pool[own.cuda()] = part
    held = [[_f64(t.transpose(1, 2).reshape(n * page, kv_heads, dim)[:length]) for t in x]]
    table = own.to(torch.int32).view(1, n).cuda()
    lens = torch.tensor([length], dtype=torch.int32).cuda()
    for new in (1, 200):
        q = _rand(torch, 13, new, 16, dim, dtype="bf16")
        out = cq.cq_attn_paged(q, *pools, table, lens, length,
                               q_starts=torch.tensor([0, new], dtype=torch.int32).cuda(), max_q=new)
        ref, mag = _attn_ref(_f64(q), held, [new], dim**-0.5)
        _within(out, ref, U["bf16"] * np.abs(ref) + (U["bf16"] + FP32) * mag + TINY, "far pages")
    # and the append reaches them
    qkv = _rand(torch, 14, 2, 16 + 2 * kv_heads, dim, dtype="bf16")
    slots = torch.tensor([pages * page - 1, 5], dtype=torch.int32).cuda()
    cq.cq_rope_append(qkv[:, :16], qkv[:, 16:24], qkv[:, 24:], None, None, None, slots, *pools)
    assert torch.equal(pools[0][-1, :, -1], qkv[0, 16:24]) and torch.equal(pools[1][0, :, 5], qkv[1, 24:])


# ---------------------------------------------------------------- shared prefix


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,page", [(2, 2, 16), (8, 2, 32), (7, 1, 64)])
@pytest.mark.parametrize("prefix,new,lens", [
    (33, [1, 1, 1], [5, 0, 70]), (500, [1] * 20, list(range(0, 60, 3))), (1, [1], [1]), (0, [1, 1], [3, 40]),
    (130, [3, 1, 40], [3, 20, 50]), (64, [1] * 150, [k % 37 for k in range(150)]),
])
def test_attn_shared_prefix(torch_dev, dtype, dim, heads, kv_heads, page, prefix, new, lens):
    torch, cq = torch_dev, _cq()
    say("shared", dtype, dim, heads, kv_heads, page, prefix, len(new))
    caches, tables, held = _paged(torch, 21, [prefix] + lens, page, kv_heads, dim, dtype)
    q = _rand(torch, 22, sum(new), heads + 2 * kv_heads, dim, dtype=dtype, scale=1.5)[:, :heads]
    starts = None
    if max(new) > 1:
        starts = torch.tensor(np.cumsum([0] + new), dtype=torch.int32).cuda()
    for opt in (dict(), dict(softcap=4.0, scale=0.2)):
        out = cq.cq_attn_shared_prefix(q, *caches, tables[0].contiguous(), prefix, tables[1:].contiguous(),
                                       torch.tensor(lens, dtype=torch.int32).cuda(), max(lens), q_starts=starts,
                                       max_q=max(new), **opt)
        ref, mag = _attn_ref(_f64(q), held[1:], new, opt.get("scale", dim**-0.5), softcap=opt.get("softcap", 0.0),
                             prefix=held[0])
        u = U[dtype]
        _within(out, ref, u * np.abs(ref) + (u + FP32) * mag + TINY, "shared prefix")


def test_attn_shared_prefix_without_own_tokens(torch_dev):
    torch, cq = torch_dev, _cq()
    caches, tables, held = _paged(torch, 23, [90], 16, 2, 64, "bf16")
    q = _rand(torch, 24, 6, 4, 64, dtype="bf16")
    lens = torch.zeros((6,), dtype=torch.int32, device="cuda")
    none = torch.empty((6, 0), dtype=torch.int32, device="cuda")
    out = cq.cq_attn_shared_prefix(q, *caches, tables[0].contiguous(), 90, none, lens, 0)
    empty = [[np.zeros((0, 2, 64))] * 2] * 6
    ref, mag = _attn_ref(_f64(q), empty, [1] * 6, 0.125, prefix=held[0])
    _within(out, ref, U["bf16"] * np.abs(ref) + (U["bf16"] + FP32) * mag + TINY, "prefix alone")


@pytest.mark.parametrize("opt", [dict()] + OPTIONS, ids=str)
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("bf16", 256), ("fp16", 256)])
@pytest.mark.parametrize("new,lens", [
    ([70, 33, 1, 64, 20], [1700, 40, 900, 64, 1290]),       # tokens of a few row tiles split many ways
    ([20, 5, 90, 1, 17], [1030, 4, 2000, 1, 17]),           # the bias's and the window's sequence not the longest
])
def test_attn_scores_and_masks_over_split_tokens(torch_dev, opt, dtype, dim, new, lens):
    import ctypes
    cq = _cq()
    # the tokens are split: the call needs room for parts
    c = cq.block.cq_kv_cache(dtype=0, kv_heads=2, dim=dim, page=16, pages=1000, k=4096, v=4096)
    a = cq.block.cq_attn_args(q=4096, out=4096, q_stride=4 * dim, tokens=sum(new), heads=4, batch=5, q_starts=4096,
                              tables=4096, table_width=200, max_q=max(new), max_kv=max(lens), kv_lens=4096, scale=1.0)
    assert cq.lib().cq_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(a)) >= 2 * sum(new) * 4 * dim * 4
    _check_attn(torch_dev, dtype, dim, 4, 2, 16, new, lens, **opt)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("bf16", 256)])
@pytest.mark.parametrize("prefix,new,lens", [(1900, [1] * 9, [0, 1, 40, 3, 300, 17, 16, 64, 5]),
                                             (1500, [90, 1, 1, 33, 0, 2], [1200, 7, 0, 33, 5, 600])])
@pytest.mark.parametrize("softcap", [0.0, 6.0])
def test_attn_shared_prefix_over_split_tokens(torch_dev, dtype, dim, prefix, new, lens, softcap):
    torch, cq = torch_dev, _cq()
    say("shared split", dtype, dim, prefix, new, lens, softcap)
    heads, kv_heads = 4, 2
    caches, tables, held = _paged(torch, 25, [prefix] + lens, 32, kv_heads, dim, dtype)
    q = _rand(torch, 26, sum(new), heads + 2 * kv_heads, dim, dtype=dtype, scale=1.5)[:, :heads]
    starts = torch.tensor(np.cumsum([0] + new), dtype=torch.int32).cuda()
    out = cq.cq_attn_shared_prefix(q, *caches, tables[0].contiguous(), prefix, tables[1:].contiguous(),
                                   torch.tensor(lens, dtype=torch.int32).cuda(), max(lens), q_starts=starts,
                                   max_q=max(new), softcap=softcap)
    ref, mag = _attn_ref(_f64(q), held[1:], new, dim**-0.5, softcap=softcap, prefix=held[0])
    _within(out, ref, U[dtype] * np.abs(ref) + (U[dtype] + FP32) * mag + TINY, "split prefix")


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("fp16", 256)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_attn_hidden_tokens_of_split_sequences_may_hold_anything(torch_dev, dtype, dim, bad):
    # a bad value that only the last query sees, and one that only the first one's window holds
    torch, cq = torch_dev, _cq()
    say("split hidden", dtype, dim, bad)
    heads, kv_heads, page, new, length = 4, 2, 16, 70, 1700
    caches, tables, held = _paged(torch, 27, [length], page, kv_heads, dim, dtype, garbage=bad)
    q = _rand(torch, 28, new, heads, dim, dtype=dtype)
    starts = torch.tensor([0, new], dtype=torch.int32).cuda()
    lens = torch.tensor([length], dtype=torch.int32).cuda()
    for window, at, hit in ((0, length - 1, new - 1), (900, length - new - 899, 0)):
        pools = [c.clone() for c in caches]
        ref, mag = _attn_ref(_f64(q), held, [new], dim**-0.5, window=window)
        pools[1][int(tables[0, at // page]), :, at % page] = bad
        out = cq.cq_attn_paged(q, *pools, tables, lens, length, q_starts=starts, max_q=new, window=window)
        rest = [i for i in range(new) if i != hit]
        _within(out[rest], ref[rest], U[dtype] * np.abs(ref[rest]) + (U[dtype] + FP32) * mag[rest] + TINY, "others")
        assert not bool(torch.isfinite(out[hit]).any())


# ---------------------------------------------------------------- streams, graphs, repeats


def _block(torch, seed):
    """Inputs of a norm, an append and an attention over what was appended."""
    heads, kv_heads, dim, page, batch = 8, 2, 64, 16, 5
    caches, tables, held = _paged(torch, seed, [60, 9, 200, 33, 1], page, kv_heads, dim, "bf16")
    lens = torch.tensor([60, 9, 200, 33, 1], dtype=torch.int32).cuda()
    last = (lens - 1).long()
    slots = (tables[torch.arange(batch).cuda(), last // page].long() * page + last % page).to(torch.int32)
    qkv = _rand(torch, seed + 1, batch, heads + 2 * kv_heads, dim, dtype="bf16")
    angle = torch.arange(256 * 32, device="cuda").view(256, 32) * 0.01
    x = _rand(torch, seed + 2, batch, heads * dim, dtype="bf16")
    w = _rand(torch, seed + 3, heads * dim, dtype="bf16")
    return caches, tables, lens, slots, qkv, angle.cos(), angle.sin(), x, w


def _run_block(cq, inputs, stream=None):
    caches, tables, lens, slots, qkv, cos, sin, x, w = inputs
    q = cq.cq_rope_append(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], cos, sin, (lens - 1), slots, *caches, stream=stream)
    o = cq.cq_attn_paged(q, *caches, tables, lens, 200, stream=stream)
    s = cq.cq_attn_shared_prefix(q, *caches, tables[2].contiguous(), 150, tables, lens, 200, stream=stream)
    h, r = cq.cq_norm_residual(x, w, 1e-5, y=o.view(o.shape[0], -1), post_weight=w, stream=stream)
    return o, s, h, r


def test_block_repeats_bit_for_bit_and_on_another_stream(torch_dev):
    torch, cq = torch_dev, _cq()
    inputs = _block(torch, 31)
    first = [t.clone() for t in _run_block(cq, inputs)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = _run_block(cq, inputs)
    side.synchronize()
    for a, b, c in zip(first, other, _run_block(cq, inputs)):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_attn_workspace_is_allocated_on_the_stream_of_the_call(torch_dev, monkeypatch):
    # else the allocator gives it to the current stream's next tensor while the
    # kernels on the other stream still write to it
    torch, cq = torch_dev, _cq()
    inputs = _block(torch, 71)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    empty, at = torch.empty, []

    def seen(*args, **kw):
        if kw.get("dtype") == torch.uint8:
            at.append(torch.cuda.current_stream())
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", seen)
    qkv, caches, tables, lens = inputs[4], inputs[0], inputs[1], inputs[2]
    got = cq.cq_attn_shared_prefix(qkv[:, :8], *caches, tables[2].contiguous(), 150, tables, lens, 200, stream=side)
    monkeypatch.undo()
    side.synchronize()
    plain = cq.cq_attn_shared_prefix(qkv[:, :8], *caches, tables[2].contiguous(), 150, tables, lens, 200)
    assert torch.equal(got, plain)
    assert at == [side]


def test_buffers_let_go_on_another_stream_are_not_handed_to_the_current_one(torch_dev):
    # the last norm of a model: its residual is let go while the kernel still writes it
    torch, cq = torch_dev, _cq()
    x, y = (_rand(torch, 81 + i, 700, 4096, dtype="bf16") for i in range(2))
    w = _rand(torch, 83, 4096, dtype="bf16")
    want, _ = cq.cq_norm_residual(x, w, 1e-5, y=y)
    x8_want, dx_want, _ = cq.cq_norm_residual_a8(x, w, 1e-5, y=y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h, r = cq.cq_norm_residual(x, w, 1e-5, y=y, stream=side)
    x8, dx, r8 = cq.cq_norm_residual_a8(x, w, 1e-5, y=y, stream=side)
    at = {r.data_ptr(), r8.data_ptr()}
    del r, r8
    others = [torch.zeros_like(x) for _ in range(4)]
    assert not at & {t.data_ptr() for t in others}
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(h, want) and torch.equal(x8, x8_want) and torch.equal(dx, dx_want)


def test_block_in_a_graph(torch_dev):
    torch, cq = torch_dev, _cq()
    inputs = _block(torch, 41)
    _run_block(cq, inputs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _run_block(cq, inputs)
    for seed in (51, 52, 53):
        fresh = _block(torch, seed)
        for i in (4, 7):
            inputs[i].copy_(fresh[i])
        want = [t.clone() for t in _run_block(cq, inputs)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_calls_on_a_side_stream_in_a_graph(torch_dev):
    torch, cq = torch_dev, _cq()
    inputs = _block(torch, 43)
    _run_block(cq, inputs)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        outs = _run_block(cq, inputs, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for seed in (54, 55, 56):
        fresh = _block(torch, seed)
        for i in (4, 7):
            inputs[i].copy_(fresh[i])
        want = [t.clone() for t in _run_block(cq, inputs)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_attn_workspace_of_the_caller(torch_dev):
    torch, cq = torch_dev, _cq()
    caches, tables, held = _paged(torch, 61, [3000, 10], 16, 2, 128, "bf16")
    q = _rand(torch, 62, 2, 8, 128, dtype="bf16")
    lens = torch.tensor([3000, 10], dtype=torch.int32).cuda()
    need = cq.cq_attn_workspace_bytes(q, *caches, tables, lens, 3000)
    want = cq.cq_attn_paged(q, *caches, tables, lens, 3000)
    # whatever the workspace holds, the result is the same
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(cq.cq_attn_paged(q, *caches, tables, lens, 3000, workspace=ws), want)
    if need > 0:
        with pytest.raises(cq.CQError) as e:
            cq.cq_attn_paged(q, *caches, tables, lens, 3000, workspace=ws[:need - 16])
        assert e.value.status == 2


# ---------------------------------------------------------------- the whole block


@pytest.mark.parametrize("a8", [False, True])
def test_decoder_block_example(torch_dev, a8):
    # Two blocks, each with about eight roundings to BF16 between FP32 steps, 2^-9
    # of the value in the mean: 2^-9 sqrt(16) < 1e-2.  Dynamic-A8 rounds the normed
    # stream to 127 steps of its largest value, a few hundredths of a product's norm.
    from examples.decoder_block import serve
    errors = serve(prompts=(37, 5, 130), tokens=3, samples=5, a8=a8)
    say("decoder block", a8, errors)
    assert len(errors) == 8 and max(errors) < (5e-2 if a8 else 1e-2)


# ---------------------------------------------------------------- caps of any size


def _f32(x):
    return float(np.float32(x))


@pytest.mark.parametrize("cap", [1e-3, 0.7, 64.0, 65.0, 1e3, 1e5, 1e6, 1e8, 1e30, 3e38])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("fp16", 256)])
@pytest.mark.parametrize("new,lens", [([1, 1, 1], [1, 40, 290]), ([90, 64], [130, 64])])
def test_attn_caps_far_from_the_scores(torch_dev, cap, dtype, dim, new, lens):
    # a cap far above the scores leaves them as they are
    _check_attn(torch_dev, dtype, dim, 4, 2, 16, new, lens, softcap=_f32(cap))


@pytest.mark.parametrize("cap", [30.0, 70.0, 200.0])
@pytest.mark.parametrize("dtype,new,lens", [("fp16", [1, 1, 1], [1, 40, 290]), ("bf16", [90, 64], [130, 64])])
def test_attn_scores_around_the_cap(torch_dev, cap, dtype, new, lens):
    # scores of up to about 70, on both sides of the cap
    _check_attn(torch_dev, dtype, 64, 4, 2, 16, new, lens, softcap=cap, scale=1.0)


@pytest.mark.parametrize("cap", [1e-37, 1e-40])
@pytest.mark.parametrize("new,length", [(1, 40), (70, 90)])
def test_attn_of_no_query_under_the_smallest_caps(torch_dev, cap, new, length):
    # a score of zero stays zero: the mean of the visible values
    torch, cq = torch_dev, _cq()
    caches, tables, held = _paged(torch, 7, [length], 16, 1, 64, "fp16")
    q = torch.zeros((new, 2, 64), dtype=torch.float16, device="cuda")
    lens = torch.tensor([length], dtype=torch.int32).cuda()
    starts = torch.tensor([0, new], dtype=torch.int32).cuda()
    out = cq.cq_attn_paged(q, *caches, tables, lens, length, q_starts=starts, max_q=new, softcap=_f32(cap))
    ref, mag = _attn_ref(_f64(q), held, [new], 0.125)
    _within(out, ref, U["fp16"] * np.abs(ref) + (U["fp16"] + FP32) * mag + TINY, "equal weights")


def test_attn_splits_of_the_longest_sequence(torch_dev):
    # 2^30 tokens of two pages, each of them repeated: 64 splits of 2^25 tiles, the
    # last split the only one with the second page's, whose keys are far above the
    # others'.  All of its tokens are alike, so that the sums are of ones.
    torch, cq = torch_dev, _cq()
    heads, dim, page = 33, 256, 1024
    k = torch.zeros((2, 1, page, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[1, ..., 0] = 100.0
    v[0], v[1] = 1.0, 2.0
    width = (1 << 30) // page
    table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
    table[0, -(width // 64):] = 1
    q = torch.zeros((1, heads, dim), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    lens = torch.tensor([1 << 30], dtype=torch.int32, device="cuda")
    say("longest sequence", lens.item())
    out = cq.cq_attn_paged(q, k, v, table, lens, 1 << 30, scale=1.0)
    assert bool((out == 2.0).all())


# ---------------------------------------------------------------- weights and their sum


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new,lens", [([1] * 6, [40, 33, 90, 17, 300, 64]), ([3, 4], [50, 200]), ([1], [1500]),
                                      ([70, 33], [100, 33]), ([40], [1500])])
@pytest.mark.parametrize("prefix", [0, 75])
def test_attn_of_equal_values_is_that_value(torch_dev, dtype, dim, new, lens, prefix):
    # Every token has the same value, the largest below 2: the output is it times
    # (sum of the weights that multiply it) / (sum that divides), and 2^-12 (FP16) or
    # 2^-9 (BF16) away from it lies the middle of its neighbour.  FP32 sums of 1500
    # terms stay within 2^-13, BF16 weights in two parts within 2^-17.  All tokens
    # but each page's first have one key, so that their weights share a rounding.
    torch, cq = torch_dev, _cq()
    say("equal values", dtype, dim, new, lens, prefix)
    heads, kv_heads, page = 8, 2, 16
    caches, tables, held = _paged(torch, 8, [max(prefix, 1)] + lens, page, kv_heads, dim, dtype)
    value = 2.0 - 2.0 * U[dtype]
    caches[0].zero_()
    caches[0][..., 0] = -1.0
    caches[0][:, :, 0, 0] = 1.0
    caches[1].fill_(value)
    q = torch.zeros((sum(new), heads, dim))
    q[..., 0] = torch.rand(q.shape[:2], generator=torch.Generator().manual_seed(4)) - 0.5
    q = q.to(_dtype(torch, dtype)).cuda()
    starts = torch.tensor(np.cumsum([0] + new), dtype=torch.int32).cuda()
    args = (tables[1:].contiguous(), torch.tensor(lens, dtype=torch.int32).cuda(), max(lens))
    kw = dict(q_starts=starts, max_q=max(new), scale=1.0)
    if prefix:
        out = cq.cq_attn_shared_prefix(q, *caches, tables[0].contiguous(), prefix, *args, **kw)
    else:
        out = cq.cq_attn_paged(q, *caches, *args, **kw)
    assert bool((out == value).all()), float((out.float() - value).abs().max())


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 4, 1), (128, 8, 2), (256, 12, 1), (64, 24, 1)])
def test_attn_weights_of_few_bf16_rows_keep_two_parts(torch_dev, dim, heads, kv_heads):
    # Values of +1 and -1 in turn under weights that nearly cancel: the output is far
    # below sum(p |v|) = 1, so that its own rounding hides nothing.  Weights in two
    # parts are within 2^-17 of themselves; in one part they would be off by 2^-9.
    torch, cq = torch_dev, _cq()
    lens, page = [2, 4, 6, 8, 32, 33, 200], 16
    say("two parts", dim, heads, kv_heads)
    caches, tables, held = _paged(torch, 9, lens, page, kv_heads, dim, "bf16")
    caches[0].mul_(0.25)
    caches[1][:, :, 0::2], caches[1][:, :, 1::2] = 1.0, -1.0
    for k, v in held:
        k *= 0.25
        v[0::2], v[1::2] = 1.0, -1.0
    q = _rand(torch, 10, len(lens), heads, dim, dtype="bf16")
    out = cq.cq_attn_paged(q, *caches, tables, torch.tensor(lens, dtype=torch.int32).cuda(), max(lens))
    ref, mag = _attn_ref(_f64(q), held, [1] * len(lens), dim**-0.5)
    _within(out, ref, U["bf16"] * np.abs(ref) + FP32 * mag, "two parts")


# ---------------------------------------------------------------- more workgroups than 32 bits of threads


def test_norm_of_more_rows_than_a_grid_has_along_x(torch_dev):
    torch, cq = torch_dev, _cq()
    rows = (1 << 26) + 5
    say("norm", rows)
    pattern = _rand(torch, 91, 1 << 13, 8, dtype="bf16")
    r = pattern.repeat((rows >> 13) + 1, 1)[:rows]
    w = _rand(torch, 92, 8, dtype="bf16")
    want, _ = cq.cq_norm_residual(pattern, w, 1e-5)
    h, _ = cq.cq_norm_residual(r, w, 1e-5, out=torch.zeros_like(r))
    assert torch.equal(h[:rows - 5].view(-1, 1 << 13, 8), want.expand(rows >> 13, -1, -1))
    assert torch.equal(h[-5:], want[:5])


def test_append_of_more_tokens_than_a_grid_has_along_x(torch_dev):
    torch, cq = torch_dev, _cq()
    tokens = (1 << 26) + 3
    say("append", tokens)
    q = torch.empty((tokens, 1, 64), dtype=torch.bfloat16, device="cuda")
    q.view(-1, 64).copy_(torch.arange(tokens, device="cuda", dtype=torch.int32).remainder(251)[:, None] + 1)
    slots = torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
    slots[-1] = 7
    caches = [torch.zeros((1, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out = cq.cq_rope_append(q, q, q, None, None, None, slots, *caches, q_out=torch.zeros_like(q))
    assert torch.equal(out, q)
    for c in caches:
        assert torch.equal(c[0, 0, 7], q[-1, 0]) and int(c.count_nonzero()) == 64
    del q, out, slots
    torch.cuda.empty_cache()


def test_attn_joins_more_rows_than_a_grid_has_along_x(torch_dev):
    # 2^20 sequences of one query behind one prefix, 64 heads: 2^26 rows, which repeat
    torch, cq = torch_dev, _cq()
    batch, heads, dim, repeat = (1 << 20) + 4, 64, 64, 1 << 10
    say("join", batch, heads)
    caches, tables, held = _paged(torch, 93, [40], 16, 1, dim, "bf16")
    few = _rand(torch, 94, repeat, heads, dim, dtype="bf16")
    q = few.repeat(batch // repeat + 1, 1, 1)[:batch]
    none = torch.empty((batch, 0), dtype=torch.int32, device="cuda")
    lens = torch.zeros((batch,), dtype=torch.int32, device="cuda")
    out = cq.cq_attn_shared_prefix(q, *caches, tables[0].contiguous(), 40, none, lens, 0, out=torch.zeros_like(q))
    ref, mag = _attn_ref(_f64(few), [[np.zeros((0, 1, dim))] * 2] * repeat, [1] * repeat, dim**-0.5, prefix=held[0])
    u = U["bf16"]
    _within(out[:repeat], ref, u * np.abs(ref) + (u + FP32) * mag + TINY, "first rows")
    for i in range(repeat, batch, repeat):
        n = min(repeat, batch - i)
        assert torch.equal(out[i:i + n], out[:n]), i
    del q, out, none, lens
    torch.cuda.empty_cache()
