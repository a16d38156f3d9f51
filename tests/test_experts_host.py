"""Host-side checks of the operators of a mixture-of-experts layer (no GPU): every bad
argument is refused, by its status, before any device work."""
import contextlib
import ctypes
import os
import random
import subprocess

import pytest

import paper_2608_06763_amd as cq
from paper_2608_06763_amd import experts as E
from tests._cases import W8_DENSE, W8_ROUTED

OK, BAD = 4096, 4100  # a 16-byte aligned address that nothing reads, and one that is not aligned
ODD = 4097


def ref(x):
    return ctypes.byref(x)


def route(**kw):
    a = dict(logits=OK, bias=OK, live=OK, chosen=OK, weights=OK, plan=OK, tokens=5, stride=64, dtype=0, experts=64,
             top=8, scoring=0, groups=4, kept_groups=2, group_top=2, renormalize=1, scale=1.0)
    a.update(kw)
    return E.cq_route_args(**a)


@pytest.mark.parametrize("kw,want", [({f: None}, 1) for f in ("logits", "chosen", "weights")] + [
    (dict(tokens=0), 1), (dict(experts=0), 1), (dict(top=0), 1), (dict(scoring=2), 1), (dict(scoring=-1), 1),
    (dict(renormalize=2), 1), (dict(groups=0), 1), (dict(kept_groups=0), 1), (dict(kept_groups=5), 1),
    (dict(group_top=0), 1), (dict(group_top=3), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(dtype=3), 6), (dict(dtype=-1), 6), (dict(experts=1028, stride=1028), 2), (dict(top=33), 2),
    (dict(experts=4, top=5), 2), (dict(groups=3), 2), (dict(groups=128, experts=256, stride=256), 2),
    (dict(stride=63), 2), (dict(stride=1 << 45), 2), (dict(tokens=1 << 28), 2),
] + [({f: BAD}, 3) for f in ("logits", "bias")] + [({f: ODD}, 3) for f in ("live", "chosen", "weights", "plan")])
def test_route_refusals(kw, want):
    L = cq.lib()
    assert L.cq_route(ref(route(**kw)), OK, 1 << 40, None) == want
    assert L.cq_route_workspace_bytes(ref(route(**kw))) == -1


def test_route_workspaces():
    L = cq.lib()
    assert L.cq_route(None, OK, 1 << 40, None) == 1 and L.cq_route_workspace_bytes(None) == -1
    few, many = route(), route(tokens=50000)
    assert L.cq_route_workspace_bytes(ref(few)) == 0
    assert L.cq_route_workspace_bytes(ref(route(tokens=50000, plan=None))) == 0
    need = L.cq_route_workspace_bytes(ref(many))
    assert 0 < need < 1 << 24
    assert L.cq_route(ref(many), None, need, None) == 1
    assert L.cq_route(ref(many), OK, need - 1, None) == 2
    assert L.cq_route(ref(many), BAD, need, None) == 3


def test_plan_refusals():
    L = cq.lib()
    need = L.cq_route_plan_workspace_bytes(400000, 64)
    assert 0 < need < 1 << 24 and L.cq_route_plan_workspace_bytes(100, 64) == 0
    assert L.cq_route_plan_workspace_bytes(0, 64) == L.cq_route_plan_workspace_bytes(5, 0) == -1
    assert L.cq_route_plan_workspace_bytes(5, 1025) == -1
    for args, want in [((None, 400000, 64, OK, OK, need), 1), ((OK, 400000, 64, None, OK, need), 1),
                       ((OK, 0, 64, OK, OK, need), 1), ((OK, 400000, 0, OK, OK, need), 1),
                       ((OK, 1 << 31, 64, OK, OK, need), 2), ((OK, 400000, 1025, OK, OK, need), 2),
                       ((ODD, 400000, 64, OK, OK, need), 3), ((OK, 400000, 64, ODD, OK, need), 3),
                       ((OK, 400000, 64, OK, None, need), 1), ((OK, 400000, 64, OK, OK, need - 1), 2),
                       ((OK, 400000, 64, OK, BAD, need), 3)]:
        assert L.cq_route_plan(*args, None) == want, args


def product(**kw):
    a = dict(x8=OK, dx=OK, w8=OK, dw=OK, bias=OK, y=OK, rows=9, n=40, k=64, y_dtype=0, experts=0, plan=None, routes=0,
             fan=0)
    a.update(kw)
    return E.cq_w8_args(**a)


PRODUCT = [({f: None}, 1) for f in ("x8", "dx", "w8", "dw", "y")] + [
    (dict(rows=0), 1), (dict(n=0), 1), (dict(k=0), 1), (dict(y_dtype=3), 6), (dict(k=72), 2), (dict(k=131072), 2),
    (dict(rows=1 << 31), 2), (dict(n=1 << 30), 2),
] + [({f: BAD}, 3) for f in ("x8", "dx", "w8", "dw", "bias", "y")]


@pytest.mark.parametrize("kw,want", PRODUCT + [(dict(rows=1 << 30, n=1 << 20), 2), (dict(rows=1 << 29), 2), (dict(plan=OK), 1), (dict(experts=3), 1), (dict(routes=3), 1),
                                               (dict(fan=1), 1)])
def test_product_refusals(kw, want):
    assert cq.lib().cq_gemm_w8(ref(product(**kw)), None) == want


@pytest.mark.parametrize("kw,want", PRODUCT + [
    (dict(plan=None), 1), (dict(experts=0), 1), (dict(routes=0), 1), (dict(fan=0), 1), (dict(experts=1025), 2),
    (dict(routes=1 << 31, rows=1 << 30, fan=2), 2), (dict(fan=1025), 2), (dict(routes=19), 2), (dict(plan=ODD), 3),
    (dict(n=1 << 29, k=131056), 2)])
def test_routed_product_refusals(kw, want):
    routed = dict(experts=4, plan=OK, routes=18, fan=2)
    routed.update(kw)
    assert cq.lib().cq_gemm_routed_w8(ref(product(**routed)), None) == want


def test_products_of_no_arguments():
    L = cq.lib()
    assert L.cq_gemm_w8(None, None) == L.cq_gemm_routed_w8(None, None) == 1


def gated(**kw):
    a = dict(gate=OK, up=OK, out=OK, rows=5, width=96, stride=192, dtype=0, act=0)
    a.update(kw)
    return E.cq_gated_args(**a)


@pytest.mark.parametrize("kw,want", [
    (dict(gate=None), 1), (dict(up=None), 1), (dict(out=None), 1), (dict(rows=0), 1), (dict(width=0), 1),
    (dict(act=2), 1), (dict(act=-1), 1), (dict(dtype=2), 6), (dict(width=92), 2), (dict(width=65544, stride=65544), 2),
    (dict(rows=1 << 31), 2), (dict(stride=100), 2), (dict(stride=88), 2), (dict(stride=1 << 45), 2),
] + [({f: BAD}, 3) for f in ("gate", "up", "out")])
def test_gated_refusals(kw, want):
    L = cq.lib()
    assert L.cq_gated(ref(gated(**kw)), None) == want
    if kw != dict(out=None):
        assert L.cq_gated_a8(ref(gated(**kw)), OK, OK, None) == want


def test_gated_to_carriers_refusals():
    L = cq.lib()
    assert L.cq_gated(None, None) == L.cq_gated_a8(None, OK, OK, None) == 1
    assert L.cq_gated_a8(ref(gated()), None, OK, None) == L.cq_gated_a8(ref(gated()), OK, None, None) == 1
    assert L.cq_gated_a8(ref(gated(width=72)), OK, OK, None) == 2
    assert L.cq_gated_a8(ref(gated()), BAD, OK, None) == L.cq_gated_a8(ref(gated()), OK, BAD, None) == 3


def combine(**kw):
    a = dict(y=OK, weights=OK, chosen=OK, base=OK, out=OK, tokens=5, width=64, top=4, experts=16, dtype=0, out_dtype=0,
             alpha=1.0)
    a.update(kw)
    return E.cq_combine_args(**a)


@pytest.mark.parametrize("kw,want", [({f: None}, 1) for f in ("y", "weights", "chosen", "out")] + [
    (dict(tokens=0), 1), (dict(width=0), 1), (dict(top=0), 1), (dict(experts=0), 1), (dict(alpha=float("nan")), 1),
    (dict(dtype=2), 6), (dict(out_dtype=1), 6), (dict(width=60), 2), (dict(width=65544), 2), (dict(top=33), 2),
    (dict(tokens=1 << 29), 2),
] + [({f: BAD}, 3) for f in ("y", "base", "out")] + [(dict(chosen=ODD), 3), (dict(weights=ODD), 3)])
def test_combine_refusals(kw, want):
    assert cq.lib().cq_combine(ref(combine(**kw)), None) == want


def test_combine_of_no_arguments():
    assert cq.lib().cq_combine(None, None) == 1


def test_packed_arguments_are_whole_structures():
    for packed, c in ((E._ROUTE, E.cq_route_args), (E._W8, E.cq_w8_args), (E._GATED, E.cq_gated_args),
                      (E._COMBINE, E.cq_combine_args)):
        assert packed.size == ctypes.sizeof(c)
        fields = [f for f, _ in c._fields_]
        got = c.from_buffer_copy(packed.pack(*range(1, len(fields) + 1)))
        assert [getattr(got, f) for f in fields] == list(range(1, len(fields) + 1))


def test_tensors_of_another_device_are_refused(monkeypatch):
    torch = E._torch()
    monkeypatch.setattr(E, "_device", lambda: 0)
    f, i = torch.zeros((4, 64)), torch.zeros((4, 64), dtype=torch.int8)
    h, c = f.bfloat16(), torch.zeros((4, 2), dtype=torch.int32)
    plan = torch.zeros((13,), dtype=torch.int32)
    for call in (lambda: cq.cq_route(f, 2), lambda: cq.cq_route_plan(c, 4), lambda: cq.cq_gemm_w8(i, f[0], i, f[0]),
                 lambda: cq.cq_gemm_routed_w8(i, f[0], i[None], f[:1], plan), lambda: cq.cq_gated(h, h),
                 lambda: cq.cq_gated_a8(h, h), lambda: cq.cq_combine(h, f[:2, :2], c[:2], 4)):
        with pytest.raises(ValueError):
            call()


def test_calls_given_a_stream_allocate_and_launch_there(monkeypatch):
    # as the block's calls: on the stream current, and recorded for the caller's own
    torch = E._torch()

    class Stream:
        device = torch.device("cpu")

    main, side = Stream(), Stream()
    now, made, used, launched = [main], [], [], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("workspace_bytes"):
                    return 512
                launched.append(now[-1])
                return 0
            return call

    def maker(empty):
        def make(*args, **kw):
            made.append(now[-1])
            return empty(*args, **kw)
        return make

    f, i = torch.zeros((4, 64)), torch.zeros((4, 64), dtype=torch.int8)
    h, c, plan = f.bfloat16(), torch.zeros((2, 2), dtype=torch.int32), torch.zeros((9,), dtype=torch.int32)
    v, w = torch.zeros((4,)), torch.zeros((2, 2))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(E, "lib", Library)
    monkeypatch.setattr(E, "_begin", lambda *t: 0)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: used.append((t.data_ptr(), s)))
    for where, name in ((torch, "empty_like"), (torch.Tensor, "new_empty")):
        monkeypatch.setattr(where, name, maker(getattr(where, name)))
    calls = [(4, lambda s: cq.cq_route(f, 2, stream=s)), (2, lambda s: cq.cq_route_plan(c, 4, stream=s)),
             (1, lambda s: cq.cq_gemm_w8(i, v, i, v, stream=s)),
             (1, lambda s: cq.cq_gemm_routed_w8(i, v, i.view(4, 1, 64), v.view(4, 1), plan, stream=s)),
             (1, lambda s: cq.cq_gated(h, h, stream=s)), (2, lambda s: cq.cq_gated_a8(h, h, stream=s)),
             (1, lambda s: cq.cq_combine(h, w, c, 4, stream=s))]
    for count, call in calls:
        for stream in (side, None):
            del made[:], used[:], launched[:]
            got = call(stream)
            want = side if stream else main
            assert len(made) == count and set(made) == {want} and launched == [want]
            got = {t.data_ptr() for t in (got if isinstance(got, tuple) else (got,))}
            assert got == {p for p, _ in used} and {s for _, s in used} == {main} if stream else not used


def test_arguments_of_other_shapes_and_types_are_refused(monkeypatch):
    torch = E._torch()
    monkeypatch.setattr(E, "_begin", lambda *t: 0)
    f, i = torch.zeros((4, 64)), torch.zeros((4, 64), dtype=torch.int8)
    h, c, v = f.bfloat16(), torch.zeros((2, 2), dtype=torch.int32), torch.zeros((4,))
    w, plan = torch.zeros((2, 2)), torch.zeros((9,), dtype=torch.int32)
    bank, scales = i.view(4, 1, 64), v.view(4, 1)
    bad = [
        lambda: cq.cq_route(f.t(), 2), lambda: cq.cq_route(f, 2, bias=v), lambda: cq.cq_route(f, 2, live=v[:1]),
        lambda: cq.cq_route(f, 2, chosen=c), lambda: cq.cq_route(f, 2, weights=f), lambda: cq.cq_route(f, 2, plan=plan),
        lambda: cq.cq_route_plan(c.t(), 4), lambda: cq.cq_route_plan(c.long(), 4),
        lambda: cq.cq_route_plan(c, 4, plan=plan[:8]),
        lambda: cq.cq_gemm_w8(i[:, ::2], v, i, v), lambda: cq.cq_gemm_w8(i, v[:3], i, v),
        lambda: cq.cq_gemm_w8(i, v, i[:, :32], v), lambda: cq.cq_gemm_w8(f, v, i, v),
        lambda: cq.cq_gemm_w8(i, v, i, v, bias=v), lambda: cq.cq_gemm_w8(i, v, i, v, out=h),
        lambda: cq.cq_gemm_routed_w8(i, v, bank, v, plan), lambda: cq.cq_gemm_routed_w8(i, v, bank, scales, plan.long()),
        lambda: cq.cq_gemm_routed_w8(i, v, bank, scales, plan, bias=scales),
        lambda: cq.cq_gemm_routed_w8(i, v, bank, scales, plan, out=h[:, :1]),
        lambda: cq.cq_gated(h, h[:, :32]), lambda: cq.cq_gated(h, f), lambda: cq.cq_gated(h[:, ::2], h[:, ::2]),
        lambda: cq.cq_gated(h, torch.zeros((4, 128)).bfloat16()[:, :64]), lambda: cq.cq_gated(h, h, out=f),
        lambda: cq.cq_gated_a8(h, h, x8=h), lambda: cq.cq_gated_a8(h, h, dx=f),
        lambda: cq.cq_combine(h[:3], w, c, 4), lambda: cq.cq_combine(h, w.double(), c, 4),
        lambda: cq.cq_combine(h, w, c.long(), 4), lambda: cq.cq_combine(h, w, c, 4, base=h),
        lambda: cq.cq_combine(h, w, c, 4, base=h[:2], out=f[:2]),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(AssertionError):
            call()
            print("taken:", n)
    for call in (lambda: cq.cq_route(f, 2, scoring="max"), lambda: cq.cq_gated(h, h, act="relu")):
        with pytest.raises(KeyError):
            call()
    with pytest.raises(ValueError):
        cq.cq_route(f.double(), 2)


# ---------------------------------------------------------------- offsets of a plan

_RUNS = """
#include "plan_run.h"
extern "C" void runs(int n, const int32_t *from, const int32_t *to, int32_t routes, int tile, int64_t *out) {
    for (int i = 0; i < n; ++i) {
        const cq::plan_run run = cq::run_of(from[i], to[i], routes);
        const uint32_t tiles = cq::tiles_of(run, tile);
        int64_t *o = out + 7 * i;
        o[0] = run.first; o[1] = run.count; o[2] = tiles;
        const cq::plan_run first = cq::tile_of(run, 0, tile), last = cq::tile_of(run, tiles ? tiles - 1 : 0, tile);
        o[3] = first.first; o[4] = first.count; o[5] = last.first; o[6] = last.count;
    }
}
"""


@pytest.fixture(scope="module")
def runs(tmp_path_factory):
    """The kernels' own arithmetic of a plan's offsets, with signed overflow an error."""
    where = tmp_path_factory.mktemp("plan_run")
    (where / "runs.cpp").write_text(_RUNS)
    csrc = os.path.join(os.path.dirname(cq.__file__), "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-ftrapv", "-shared", "-fPIC", "-I", csrc, "-o",
                           str(where / "runs.so"), str(where / "runs.cpp")])
    call = ctypes.CDLL(str(where / "runs.so")).runs

    def run(pairs, routes, tile):
        n, words = len(pairs), ctypes.c_int32 * len(pairs)
        out = (ctypes.c_int64 * (7 * n))()
        call(n, words(*(a for a, _ in pairs)), words(*(b for _, b in pairs)), routes, tile, out)
        return [tuple(out[7 * i:7 * i + 7]) for i in range(n)]
    return run


@pytest.mark.parametrize("tile", [16, 64, 128, 256])
@pytest.mark.parametrize("routes", [1, 2, 299, 300, 8191, 2**29])
def test_no_offsets_of_a_plan_lead_outside_its_routes(runs, routes, tile):
    far, rng = 2**31, random.Random(routes + tile)
    odd = {0, 1, 5, 16, 255, 256, 257, routes - 1, routes, routes + 1, 2 * routes, far - 1, far - 2, far - 300}
    odd = sorted({v for o in odd for v in (o, -o, -o - 1) if -far <= v < far})
    pairs = [(a, b) for a in odd for b in odd]
    pairs += [(rng.randrange(-far, far), rng.randrange(-far, far)) for _ in range(2000)]
    pairs += [(rng.randrange(0, routes + 2), rng.randrange(-far, -far + routes + 2)) for _ in range(2000)]
    for (a, b), (first, count, tiles, *ends) in zip(pairs, runs(pairs, routes, tile)):
        lo, hi = (min(max(v, 0), routes) for v in (a, b))
        assert (first, count, tiles) == (lo, max(hi - lo, 0), -(-max(hi - lo, 0) // tile)), (a, b)
        if tiles:
            last = lo + (tiles - 1) * tile
            assert ends == [lo, min(tile, hi - lo), last, hi - last] and 0 <= last < hi <= routes, (a, b)


# ---------------------------------------------------------------- kernels of the products


def test_sizes_of_the_gpu_tests_take_every_kernel():
    # a change of the choice must not leave one of them without a test unseen
    taken = {False: {want for *_, want in W8_DENSE}, True: {want for *_, want in W8_ROUTED}}
    for rows, n, k, want in W8_DENSE:
        assert cq.cq_probe_w8_kernel(rows, n, k) == want, (rows, n, k)
    for experts, tokens, top, n, k, want in W8_ROUTED:
        for rows, fan in ((tokens, top), (tokens * top, 1)):
            assert cq.cq_probe_w8_kernel(rows, n, k, experts, tokens * top, fan) == want, (experts, tokens, top, n, k)
    few, tiles = {("few", 16, w, 4) for w in (16, 32, 64)}, {(128, 128, 2), (128, 128, 4), (128, 256, 3), (256, 256, 2)}
    assert taken[False] == few | {("rows", 16, 32, 3), ("rows", 16, 64, 3), ("rows", 32, 32, 2)} | {
        ("tiles", *t) for t in tiles | {(64, 128, 4)}}
    assert taken[True] == few | {("tiles", *t) for t in tiles | {(64, 128, 2), (64, 128, 4), (64, 256, 2)}}
    for rows in (1, 3, 8, 9, 16, 17, 40, 64, 65, 130, 300, 700, 1300, 3000, 8191):
        for n in (1, 40, 300, 1001, 2003, 4096, 6144, 12001, 28672):
            for k in (16, 144, 1040, 2064, 4112, 8192, 14336, 131056):
                assert cq.cq_probe_w8_kernel(rows, n, k) in taken[False], (rows, n, k)
                for experts in (1, 8, 48, 128, 1000):
                    if rows * k < 1 << 31:
                        assert cq.cq_probe_w8_kernel(rows, n, k, experts, rows) in taken[True], (rows, n, k, experts)


def test_kernels_of_products_that_are_refused():
    L, tile = cq.lib(), (ctypes.c_int32 * 3)()
    assert cq.cq_probe_w8_kernel(5, 40, 17) is None and cq.cq_probe_w8_kernel(5, 40, 16, 4, 6, 1) is None
    assert cq.cq_probe_w8_kernel(65536, 203, 32768, 5, 131072, 2) == ("tiles far", 128, 128, 2)
    assert cq.cq_probe_w8_kernel(65535, 203, 32768, 5, 131070, 2)[0] == "tiles"
    assert L.cq_probe_w8_kernel(None, 0, tile) == 0 and L.cq_probe_w8_kernel(ref(product()), 0, None) == 0
    assert L.cq_probe_w8_kernel(ref(product()), 0, tile) == 2 and L.cq_probe_w8_kernel(ref(product()), 1, tile) == 0
