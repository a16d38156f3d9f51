"""Host-side checks of the operators between the packed products (no GPU): every
bad argument is refused, by its status, before any device work."""
import ctypes

import pytest

import paper_2608_06763_amd as cq
from paper_2608_06763_amd.block import cq_attn_args, cq_kv_cache, cq_norm_args, cq_rope_args

OK, BAD = 4096, 4100  # a 16-byte aligned address that nothing reads, and one that is not aligned


def ref(x):
    return ctypes.byref(x)


def norm(**kw):
    a = dict(y=OK, post_weight=OK, gate=OK, residual=OK, weight=OK, residual_out=OK, out=OK, gate_stride=64, rows=3,
             width=64, dtype=0, residual_dtype=0, alpha=1.0, eps=1e-5, weight_offset=0.0)
    a.update(kw)
    return cq_norm_args(**a)


@pytest.mark.parametrize("kw,want", [
    (dict(residual=None), 1), (dict(weight=None), 1), (dict(out=None), 1), (dict(rows=0), 1), (dict(width=0), 1),
    (dict(y=None), 1), (dict(y=None, post_weight=None), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(alpha=float("inf")), 1), (dict(weight_offset=float("nan")), 1), (dict(width=60), 2), (dict(width=32776), 2),
    (dict(rows=1 << 31), 2), (dict(gate_stride=56), 2), (dict(gate_stride=68), 2), (dict(gate_stride=-64), 2),
    (dict(gate_stride=1 << 41), 2), (dict(dtype=2), 6), (dict(residual_dtype=1), 6), (dict(residual_dtype=5), 6),
] + [({f: BAD}, 3) for f in ("y", "post_weight", "gate", "residual", "weight", "residual_out", "out")])
def test_norm_refusals(kw, want):
    L = cq.lib()
    assert L.cq_norm_residual(ref(norm(**kw)), None) == want
    if kw != dict(out=None):
        assert L.cq_norm_residual_a8(ref(norm(**kw)), OK, OK, None) == want


def test_norm_a8_refusals():
    L = cq.lib()
    assert L.cq_norm_residual(None, None) == 1
    assert L.cq_norm_residual_a8(ref(norm()), None, OK, None) == 1
    assert L.cq_norm_residual_a8(ref(norm()), OK, None, None) == 1
    assert L.cq_norm_residual_a8(ref(norm(width=72, gate_stride=72)), OK, OK, None) == 2
    assert L.cq_norm_residual_a8(ref(norm()), BAD, OK, None) == 3
    assert L.cq_norm_residual_a8(ref(norm()), OK, BAD, None) == 3


def cache(**kw):
    a = dict(dtype=0, kv_heads=2, dim=64, page=16, pages=10, k=OK, v=OK)
    a.update(kw)
    return cq_kv_cache(**a)


BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(kv_heads=0), 1), (dict(pages=0), 1), (dict(dtype=2), 6),
              (dict(dim=96), 8), (dict(dim=32), 8), (dict(page=8), 2), (dict(page=48), 2), (dict(page=2048), 2),
              (dict(pages=1 << 27), 2), (dict(kv_heads=70000), 2), (dict(k=BAD), 3), (dict(v=BAD), 3)]


def rope(**kw):
    a = dict(q=OK, k=OK, v=OK, q_out=OK, q_stride=256, k_stride=128, v_stride=128, q_out_stride=256, cos=OK, sin=OK,
             positions=OK, slots=OK, tokens=5, table_rows=9, heads=4, rot=64, interleaved=0)
    a.update(kw)
    return cq_rope_args(**a)


ROPE_POINTERS = ("q", "k", "v", "q_out", "cos", "sin", "positions", "slots")


@pytest.mark.parametrize("kw,want", [({f: None}, 1) for f in ROPE_POINTERS] + [
    (dict(tokens=0), 1), (dict(heads=0), 1), (dict(table_rows=0), 1), (dict(interleaved=2), 1), (dict(rot=-16), 1),
    (dict(rot=80), 2), (dict(rot=24), 2), (dict(tokens=1 << 31), 2), (dict(q_stride=248), 2), (dict(q_stride=260), 2),
    (dict(k_stride=120), 2), (dict(v_stride=132), 2), (dict(q_out_stride=264), 2), (dict(q_stride=1 << 41), 2),
] + [({f: BAD}, 3) for f in ("q", "k", "v", "q_out", "cos", "sin")] + [({f: 4097}, 3) for f in ("positions", "slots")])
def test_rope_refusals(kw, want):
    L = cq.lib()
    assert L.cq_rope_append(ref(cache()), ref(rope(**kw)), None) == want


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_cache_refusals(kw, want):
    L = cq.lib()
    assert L.cq_rope_append(ref(cache(**kw)), ref(rope()), None) == want
    assert L.cq_attn_paged(ref(cache(**kw)), ref(attn()), OK, 1 << 40, None) == want
    assert L.cq_attn_workspace_bytes(ref(cache(**kw)), ref(attn())) == -1


def attn(**kw):
    a = dict(q=OK, out=OK, q_stride=512, tokens=7, heads=4, batch=3, q_starts=OK, tables=OK, table_width=9, max_q=4,
             max_kv=100, kv_lens=OK, scale=0.1, softcap=0.0, window=0, slopes=None, bidir=None, prefix_table=None,
             prefix_len=0)
    a.update(kw)
    return cq_attn_args(**a)


BAD_ATTN = [
    (dict(q=None), 1), (dict(out=None), 1), (dict(kv_lens=None), 1), (dict(tables=None), 1), (dict(tokens=0), 1),
    (dict(batch=0), 1), (dict(heads=0), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("inf")), 1),
    (dict(scale=float("nan")), 1), (dict(softcap=-1.0), 1), (dict(softcap=float("nan")), 1), (dict(max_q=0), 1),
    (dict(max_kv=-1), 1), (dict(table_width=-1), 1), (dict(heads=5), 2), (dict(q_stride=248), 2),
    (dict(q_stride=260), 2), (dict(q_stride=1 << 41), 2), (dict(tokens=1 << 31), 2), (dict(q_starts=None), 2),
    (dict(q_starts=None, tokens=3), 2), (dict(max_q=8), 2), (dict(max_kv=(1 << 30) + 1), 2),
    (dict(table_width=1 << 30), 2), (dict(q=BAD), 3), (dict(out=BAD), 3), (dict(q_starts=4097), 3),
    (dict(tables=4097), 3), (dict(kv_lens=4097), 3),
]


@pytest.mark.parametrize("kw,want", BAD_ATTN + [(dict(window=-1), 1), (dict(slopes=4097), 3), (dict(bidir=4097), 3)])
def test_attn_refusals(kw, want):
    L = cq.lib()
    assert L.cq_attn_paged(ref(cache()), ref(attn(**kw)), OK, 1 << 40, None) == want
    assert L.cq_attn_workspace_bytes(ref(cache()), ref(attn(**kw))) == -1


@pytest.mark.parametrize("kw,want", BAD_ATTN + [
    (dict(prefix_table=None), 1), (dict(prefix_len=-1), 1), (dict(prefix_len=(1 << 30) + 1), 2),
    (dict(prefix_table=4097), 3), (dict(window=5), 8), (dict(slopes=OK), 8), (dict(bidir=OK), 8)])
def test_shared_prefix_refusals(kw, want):
    L = cq.lib()
    a = attn(**{**dict(prefix_table=OK, prefix_len=40), **kw})
    assert L.cq_attn_shared_prefix(ref(cache()), ref(a), OK, 1 << 40, None) == want
    assert L.cq_attn_shared_prefix(ref(cache()), None, OK, 1 << 40, None) == 1


def test_attn_counts_its_work_in_31_bits():
    # 17 * 8 key heads of 2^25 units of 32 tokens
    L = cq.lib()
    c = cache(kv_heads=8, page=1024)
    a = attn(heads=8, tokens=17, batch=17, max_q=1, max_kv=1 << 30, table_width=1 << 20)
    assert L.cq_attn_paged(ref(c), ref(a), OK, 1 << 50, None) == 2
    a = attn(heads=8, tokens=7, batch=7, max_q=1, max_kv=1 << 30, table_width=1 << 20)
    assert L.cq_attn_workspace_bytes(ref(c), ref(a)) > 0


def test_attn_counts_its_workgroups_in_32_bits_of_threads():
    L = cq.lib()
    c = cache(kv_heads=8)
    # one workgroup for each sequence and key head, or few that share the tokens
    for batch, most, want in ((1 << 21, 20, 2), ((1 << 21) + 5, 20, 2), (1 << 20, 20, 0), ((1 << 21) + 5, 3000, 0)):
        a = attn(heads=8, tokens=batch, batch=batch, q_starts=None, max_q=1, max_kv=most, table_width=200)
        need = L.cq_attn_workspace_bytes(ref(c), ref(a))
        assert need >= 0 if want == 0 else need == -1
        if want:
            assert L.cq_attn_paged(ref(c), ref(a), OK, 1 << 50, None) == want


def test_paged_call_takes_no_prefix():
    L = cq.lib()
    assert L.cq_attn_paged(ref(cache()), ref(attn(prefix_table=OK, prefix_len=4)), OK, 1 << 40, None) == 1
    assert L.cq_attn_paged(None, ref(attn()), OK, 1 << 40, None) == 1


def test_workspace_refusals():
    L = cq.lib()
    a = attn(max_kv=100000, table_width=6250, tokens=3, max_q=1)
    need = L.cq_attn_workspace_bytes(ref(cache()), ref(a))
    assert need >= 0
    if need:
        assert L.cq_attn_paged(ref(cache()), ref(a), None, 0, None) == 1
        assert L.cq_attn_paged(ref(cache()), ref(a), OK, need - 1, None) == 2
        assert L.cq_attn_paged(ref(cache()), ref(a), OK + 8, need, None) == 3


def test_binding_refuses_shapes_and_types():
    import torch
    r, w = torch.zeros((3, 64)), torch.zeros((64,), dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        cq.cq_norm_residual(r, w[:32], 1e-5)
    with pytest.raises(AssertionError):
        cq.cq_norm_residual(r, w, 1e-5, y=r)  # y in another type than the weight
    with pytest.raises(AssertionError):
        cq.cq_norm_residual(r, w, 1e-5, gate=w)  # a gate of nothing
    kv = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    q, one = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3,), dtype=torch.int32)
    with pytest.raises(AssertionError):
        cq.cq_attn_paged(q, kv, kv, one.view(3, 1).long(), one, 5)
    with pytest.raises(AssertionError):
        cq.cq_attn_paged(q.half(), kv, kv, one.view(3, 1), one, 5)
    with pytest.raises(AssertionError):
        cq.cq_attn_paged(q.transpose(0, 1), kv, kv, one.view(3, 1), one, 5)
    with pytest.raises(AssertionError):
        cq.cq_rope_append(q, q, q, None, None, None, one, kv, kv)


def test_what_a_call_on_a_stream_allocates_is_that_streams(monkeypatch):
    # the library is not called: its place is taken by a list of the streams it is given
    import contextlib
    import torch
    from paper_2608_06763_amd import block

    class Stream:
        cuda_stream = 77

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
                if name == "cq_attn_workspace_bytes":
                    return 512
                launched.append(now[-1])
                return 0
            return call

    def maker(make):
        def f(*args, **kw):
            made.append(now[-1])
            return make(*args, **kw)
        return f

    r, w = torch.zeros((3, 64), dtype=torch.bfloat16), torch.zeros((64,), dtype=torch.bfloat16)
    kv = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    q, one = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3,), dtype=torch.int32)
    table = one.view(3, 1)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(block, "lib", Library)
    monkeypatch.setattr(block, "_stream_ptr", lambda stream=None: 0)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: used.append((t.data_ptr(), s)))
    for where, name in ((torch, "empty"), (torch, "empty_like"), (torch.Tensor, "new_empty")):
        monkeypatch.setattr(where, name, maker(getattr(where, name)))
    calls = [
        (4, lambda s: cq.cq_norm_residual(r, w, 1e-5, y=r, stream=s) + cq.cq_norm_residual(r, w, 1e-5, y=r, stream=s)),
        (4, lambda s: cq.cq_norm_residual_a8(r, w, 1e-5, y=r, out=r, stream=s) +
            cq.cq_norm_residual_a8(r, w, 1e-5, y=r, residual_out=r, stream=s)[:1]),
        (1, lambda s: cq.cq_rope_append(q, q[:, :2], q[:, 2:], None, None, None, one, kv, kv, stream=s)),
        (2, lambda s: cq.cq_attn_paged(q, kv, kv, table, one, 5, stream=s)),
        (2, lambda s: cq.cq_attn_shared_prefix(q, kv, kv, one, 40, table, one, 5, stream=s)),
    ]
    for least, call in calls:
        for stream in (side, None):
            del made[:], used[:], launched[:]
            got = call(stream)
            want = side if stream else main
            assert len(made) >= least and set(made) == {want} and set(launched) == {want}
            got = {t.data_ptr() for t in (got if isinstance(got, tuple) else (got,))}
            if stream:
                # the caller's stream may go on with the results, and they are nobody's before it has
                assert {s for _, s in used} == {main} and got <= {p for p, _ in used}
            else:
                assert not used
    # what the caller gave stays as it is
    del made[:], used[:]
    h, same = cq.cq_norm_residual(r, w, 1e-5, y=r, out=torch.zeros_like(r), residual_out=r, stream=side)
    assert same is r and not used and not made


def test_packed_arguments_are_whole_structures():
    # the library copies all of a structure, its padding too, from the bytes it is given
    from paper_2608_06763_amd import block
    for packed, c in ((block._NORM, cq_norm_args), (block._CACHE, cq_kv_cache), (block._ROPE, cq_rope_args),
                      (block._ATTN, block.cq_attn_args)):
        assert packed.size == ctypes.sizeof(c)
        # and every field lies where C has it
        fields = [f for f, _ in c._fields_]
        got = c.from_buffer_copy(packed.pack(*range(1, len(fields) + 1)))
        assert [getattr(got, f) for f in fields] == list(range(1, len(fields) + 1))


@pytest.mark.parametrize("prompts", [64, 128])
def test_attn_workspace_is_for_the_rows_that_there_are(prompts):
    # one chunk of 4096 tokens beside single tokens of other sequences, all behind a
    # prefix: a part of each kind for each of the call's rows, FP32 with two statistics,
    # and not the longest sequence's room for every one of them
    L = cq.lib()
    tokens, heads, dim = 4096 + prompts - 1, 32, 128
    c = cache(kv_heads=8, dim=dim, page=64, pages=100000)
    a = attn(heads=heads, q_stride=heads * dim, tokens=tokens, batch=prompts, max_q=4096, max_kv=4096, table_width=100,
             prefix_table=OK, prefix_len=1000)
    need = L.cq_attn_workspace_bytes(ref(c), ref(a))
    assert 0 < need <= 2 * tokens * heads * (4 * dim + 8) + 4096
