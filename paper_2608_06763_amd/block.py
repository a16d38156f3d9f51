"""The operators of a decoder block between its packed products (include/cq_block.h).

Arguments are device tensors; the binding only marshals them.  A paged cache is
two tensors [pages, kv_heads, page, dim] that the caller owns.  A call given a
stream runs there, and what it allocates is allocated there; the caller orders it
with the streams that made its arguments and that use its results.
"""
from __future__ import annotations

import ctypes
import struct

from . import CQ_BF16, CQ_FP16, CQ_FP32, CQError, _stream_ptr, lib

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class cq_norm_args(ctypes.Structure):
    _fields_ = [("y", _vp), ("post_weight", _vp), ("gate", _vp), ("residual", _vp), ("weight", _vp),
                ("residual_out", _vp), ("out", _vp), ("gate_stride", _i64), ("rows", _i64), ("width", _i64),
                ("dtype", _i32), ("residual_dtype", _i32), ("alpha", _f32), ("eps", _f32), ("weight_offset", _f32)]


class cq_kv_cache(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("kv_heads", _i32), ("dim", _i32), ("page", _i32), ("pages", _i64), ("k", _vp),
                ("v", _vp)]


class cq_rope_args(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("q_out", _vp), ("q_stride", _i64), ("k_stride", _i64),
                ("v_stride", _i64), ("q_out_stride", _i64), ("cos", _vp), ("sin", _vp), ("positions", _vp),
                ("slots", _vp), ("tokens", _i64), ("table_rows", _i64), ("heads", _i32), ("rot", _i32),
                ("interleaved", _i32)]


class cq_attn_args(ctypes.Structure):
    _fields_ = [("q", _vp), ("out", _vp), ("q_stride", _i64), ("tokens", _i64), ("heads", _i32), ("batch", _i32),
                ("q_starts", _vp), ("tables", _vp), ("table_width", _i32), ("max_q", _i32), ("max_kv", _i32),
                ("kv_lens", _vp), ("scale", _f32), ("softcap", _f32), ("window", _i32), ("slopes", _vp),
                ("bidir", _vp), ("prefix_table", _vp), ("prefix_len", _i64)]


# The same structures as bytes: the calls pack their arguments in one step, which
# takes a third of the time of filling a ctypes structure field by field.
_NORM = struct.Struct("@7P3q2i3f4x")
_CACHE = struct.Struct("@4iq2P")
_ROPE = struct.Struct("@4P4q4P2q3i4x")
_ATTN = struct.Struct("@2P2q2i2P3iP2fi3Pq")
for _s, _c in ((_NORM, cq_norm_args), (_CACHE, cq_kv_cache), (_ROPE, cq_rope_args), (_ATTN, cq_attn_args)):
    # to the last byte, C's padding at the end among them: calls copy whole structures
    assert _s.size == ctypes.sizeof(_c), _c


def declare(L):
    """Argument types of the entry points in a loaded library (structures by address)."""
    for name, args in (("cq_norm_residual", [_vp, _vp]),
                       ("cq_norm_residual_a8", [_vp, _vp, _vp, _vp]),
                       ("cq_rope_append", [_vp, _vp, _vp]),
                       ("cq_attn_paged", [_vp, _vp, _vp, _i64, _vp]),
                       ("cq_attn_shared_prefix", [_vp, _vp, _vp, _i64, _vp])):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = args
    L.cq_attn_workspace_bytes.restype = _i64
    L.cq_attn_workspace_bytes.argtypes = [_vp, _vp]


torch = None  # imported with the first call, as by the package
_types = {}


def _torch():
    global torch
    if torch is None:
        import torch as t
        _types.update({t.bfloat16: CQ_BF16, t.float16: CQ_FP16, t.float32: CQ_FP32})
        torch = t
    return torch


def _type(t):
    """dtype code of a tensor."""
    code = _types.get(t.dtype)
    if code is None:
        raise ValueError(f"unsupported dtype {t.dtype}")
    return code


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _dense(t, like):
    """t has the shape and type of `like` and is contiguous."""
    assert t.dtype == like.dtype and t.shape == like.shape and t.is_contiguous()
    return t.data_ptr()


def _vector(t, size, dtype):
    assert t.dtype == dtype and t.shape == (size,) and t.is_contiguous()
    return t.data_ptr()


def _on(stream, call, *args):
    """A call on a stream of the caller's: run with that stream current.

    Every buffer that the call makes is then the stream's.  The allocator hands a
    block that is let go to the next tensor of the stream that it was made on, and
    one of any other stream would not wait for the kernels.  The stream that was
    current may use what is returned as its own, so letting that go waits for it."""
    with torch.cuda.stream(stream):
        got = call(*args)
    for t in got if isinstance(got, tuple) else (got,):
        if not any(t is a for a in args):
            t.record_stream(torch.cuda.current_stream(t.device))
    return got


# ---------------------------------------------------------------- norms


def _norm_args(residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out, residual_out):
    rows, width = residual.shape
    dtype = weight.dtype
    assert residual.is_contiguous()
    y_at = post = gate_at = stride = out_at = r_at = 0
    r = residual
    if y is not None:
        assert y.dtype == dtype and y.shape == residual.shape and y.is_contiguous()
        y_at = y.data_ptr()
        if residual_out is None:
            r = torch.empty_like(residual)
            r_at = r.data_ptr()
        if post_weight is not None:
            post = _vector(post_weight, width, dtype)
        if gate is not None:
            # one gate for all rows, or a row for each
            assert gate.dtype == dtype and gate.shape[-1] == width and gate.stride(-1) == 1
            if gate.dim() == 2:
                assert gate.shape[0] == rows
                # the stride of a single row is never used: any legal one serves
                stride = gate.stride(0) if rows > 1 else width
            else:
                assert gate.dim() == 1
            gate_at = gate.data_ptr()
    else:
        assert post_weight is None and gate is None
    if residual_out is not None:
        r = residual_out
        r_at = _dense(r, residual)
    if out is not None:
        assert out.dtype == dtype and out.shape == residual.shape and out.is_contiguous()
        out_at = out.data_ptr()
    args = _NORM.pack(y_at, post, gate_at, residual.data_ptr(), _vector(weight, width, dtype), r_at, out_at, stride,
                      rows, width, _type(weight), _type(residual), alpha, eps, weight_offset)
    return args, r


def cq_norm_residual(residual, weight, eps, y=None, post_weight=None, gate=None, alpha=1.0, weight_offset=0.0,
                     out=None, residual_out=None, stream=None):
    """r' = residual + alpha * gate * (y or its post norm); h = norm(r') * weight.

    Returns (h, r').  residual [rows, width] in the model dtype or FP32; y,
    weight, post_weight [width] and gate ([width] or [rows, width]) in the model
    dtype.  Without y, r' is the residual itself, or its copy in residual_out.
    residual_out may be residual, out may be y."""
    _torch()
    if stream is not None:
        return _on(stream, cq_norm_residual, residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out,
                   residual_out)
    if out is None:
        # an empty_like that takes no dtype is twice as fast
        out = torch.empty_like(residual) if residual.dtype == weight.dtype else \
            torch.empty_like(residual, dtype=weight.dtype)
    args, r = _norm_args(residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out, residual_out)
    st = lib().cq_norm_residual(args, _stream_ptr())
    if st:
        raise CQError(st, "cq_norm_residual")
    return out, r


def cq_norm_residual_a8(residual, weight, eps, y=None, post_weight=None, gate=None, alpha=1.0, weight_offset=0.0,
                        out=None, residual_out=None, x8=None, dx=None, stream=None):
    """cq_norm_residual with h straight to the Dynamic-A8 carriers; returns
    (x8, dx, r').  h itself is written only into a given out."""
    _torch()
    if stream is not None:
        return _on(stream, cq_norm_residual_a8, residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out,
                   residual_out, x8, dx)
    rows = residual.shape[0]
    if x8 is None:
        x8 = torch.empty_like(residual, dtype=torch.int8)
    if dx is None:
        dx = torch.empty((rows,), dtype=torch.float32, device=residual.device)
    assert x8.shape == residual.shape and x8.is_contiguous() and x8.dtype == torch.int8
    args, r = _norm_args(residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out, residual_out)
    st = lib().cq_norm_residual_a8(args, x8.data_ptr(), _vector(dx, rows, torch.float32), _stream_ptr())
    if st:
        raise CQError(st, "cq_norm_residual_a8")
    return x8, dx, r


# ---------------------------------------------------------------- the paged cache


def _cache(k_cache, v_cache):
    pages, kv_heads, page, dim = k_cache.shape
    assert k_cache.is_contiguous()
    cache = _CACHE.pack(_type(k_cache), kv_heads, dim, page, pages, k_cache.data_ptr(), _dense(v_cache, k_cache))
    return cache, kv_heads, dim


def _heads_stride(x, dtype, tokens, heads, dim):
    """Stride between tokens of x [tokens, heads, dim], whose heads are dense."""
    token, head, one = x.stride()
    assert x.shape == (tokens, heads, dim) and x.dtype == dtype and one == 1 and (head == dim or heads == 1)
    # the stride of a single token is never used: any legal one serves
    return token if tokens > 1 else heads * dim


def cq_rope_append(q, k, v, cos, sin, positions, slots, k_cache, v_cache, interleaved=False, q_out=None, stream=None):
    """Rotate q and k by their positions and write k and v into their slots of
    the cache; returns the rotated queries [tokens, heads, dim].

    q, k, v [tokens, heads, dim] may be slices of one fused product; cos, sin
    FP32 [rows, rot / 2], or None for no rotation; positions, slots int32
    [tokens].  q_out may be q."""
    _torch()
    if stream is not None:
        return _on(stream, cq_rope_append, q, k, v, cos, sin, positions, slots, k_cache, v_cache, interleaved, q_out)
    cache, kv_heads, dim = _cache(k_cache, v_cache)
    tokens, heads, _ = q.shape
    dtype, int32 = k_cache.dtype, torch.int32
    q_stride = _heads_stride(q, dtype, tokens, heads, dim)
    k_stride = _heads_stride(k, dtype, tokens, kv_heads, dim)
    v_stride = _heads_stride(v, dtype, tokens, kv_heads, dim)
    if q_out is None:
        q_out = q.new_empty((tokens, heads, dim))
        out_stride = heads * dim
    else:
        out_stride = _heads_stride(q_out, dtype, tokens, heads, dim)
    rows = rot = cos_at = sin_at = at = 0
    if cos is not None:
        rows, half = cos.shape
        rot = 2 * half
        assert cos.dtype == torch.float32 and cos.is_contiguous()
        cos_at, sin_at, at = cos.data_ptr(), _dense(sin, cos), _vector(positions, tokens, int32)
    args = _ROPE.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), q_stride,
                      k_stride, v_stride, out_stride, cos_at, sin_at, at, _vector(slots, tokens, int32), tokens, rows,
                      heads, rot, interleaved)
    st = lib().cq_rope_append(cache, args, _stream_ptr())
    if st:
        raise CQError(st, "cq_rope_append")
    return q_out


def _attn(where, q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts, max_q, scale, softcap, window, slopes, bidir,
          prefix_table, prefix_len, out, workspace, stream):
    _torch()
    if stream is not None:
        return _on(stream, _attn, where, q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts, max_q, scale, softcap,
                   window, slopes, bidir, prefix_table, prefix_len, out, workspace, None)
    cache, _, dim = _cache(k_cache, v_cache)
    tokens, heads, _ = q.shape
    batch, int32 = kv_lens.shape[0], torch.int32
    stride = _heads_stride(q, k_cache.dtype, tokens, heads, dim)
    if out is None:
        out = q.new_empty((tokens, heads, dim))
    else:
        assert out.dtype == q.dtype and out.shape == q.shape and out.is_contiguous()
    sequences, width = tables.shape
    assert tables.dtype == int32 and sequences == batch and tables.is_contiguous()
    prefix_at = 0
    if prefix_table is not None:
        assert prefix_table.dtype == int32 and prefix_table.is_contiguous()
        assert prefix_len <= prefix_table.numel() * k_cache.shape[2]
        prefix_at = prefix_table.data_ptr()
    args = _ATTN.pack(
        q.data_ptr(), out.data_ptr(), stride, tokens, heads, batch,
        0 if q_starts is None else _vector(q_starts, batch + 1, int32), tables.data_ptr(), width, max_q, max_kv,
        _vector(kv_lens, batch, int32), dim**-0.5 if scale is None else scale, softcap, window,
        0 if slopes is None else _vector(slopes, heads, torch.float32),
        0 if bidir is None else _vector(bidir, batch, int32), prefix_at, prefix_len)
    L = lib()
    need = 0
    if workspace is None:
        need = L.cq_attn_workspace_bytes(cache, args)
        if need > 0:
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
    else:
        assert workspace.is_contiguous()
        need = workspace.numel() * workspace.element_size()
    st = getattr(L, where)(cache, args, _ptr(workspace), need, _stream_ptr())
    if st:
        raise CQError(st, where)
    return out


def cq_attn_paged(q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts=None, max_q=1, scale=None, softcap=0.0,
                  window=0, slopes=None, bidir=None, out=None, workspace=None, stream=None):
    """Attention of the sequences' newest tokens over the paged cache; returns
    [tokens, heads, dim].

    q [tokens, heads, dim] may be a slice of a fused product; tables int32
    [batch, width], kv_lens int32 [batch]; q_starts int32 [batch + 1], or None
    for one query of every sequence; max_q and max_kv bound the sequences.
    scale defaults to dim ** -0.5.  A workspace given by the caller
    (cq_attn_workspace_bytes) must not be shared by calls that can overlap."""
    return _attn("cq_attn_paged", q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts, max_q, scale, softcap, window,
                 slopes, bidir, None, 0, out, workspace, stream)


def cq_attn_shared_prefix(q, k_cache, v_cache, prefix_table, prefix_len, tables, kv_lens, max_kv, q_starts=None,
                          max_q=1, scale=None, softcap=0.0, out=None, workspace=None, stream=None):
    """cq_attn_paged for sequences that all begin with the prefix_len tokens of
    prefix_table (int32), which are read once; tables, kv_lens and max_kv
    describe each one's own tokens behind them."""
    return _attn("cq_attn_shared_prefix", q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts, max_q, scale,
                 softcap, 0, None, None, prefix_table, prefix_len, out, workspace, stream)


def cq_attn_workspace_bytes(q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts=None, max_q=1, prefix_len=0):
    """Bytes of workspace that an attention call of these sizes needs."""
    _torch()
    cache, _, dim = _cache(k_cache, v_cache)
    tokens, heads, _ = q.shape
    args = _ATTN.pack(q.data_ptr(), q.data_ptr(), _heads_stride(q, k_cache.dtype, tokens, heads, dim), tokens, heads,
                      kv_lens.shape[0], _ptr(q_starts), tables.data_ptr(), tables.shape[1], max_q, max_kv,
                      kv_lens.data_ptr(), 1.0, 0.0, 0, 0, 0, tables.data_ptr() if prefix_len else 0, prefix_len)
    return int(lib().cq_attn_workspace_bytes(cache, args))
