"""The operators of a decoder block between its packed products (include/cq_block.h).

Arguments are device tensors; the binding only marshals them.  A paged cache is
two tensors [pages, kv_heads, page, dim] that the caller owns.
"""
from __future__ import annotations

import ctypes

from . import CQ_BF16, CQ_FP16, CQ_FP32, _check, _dt, _stream_ptr, _torch, lib

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


def declare(L):
    """Argument types of the entry points in a loaded library."""
    P = ctypes.POINTER
    for name, args in (("cq_norm_residual", [P(cq_norm_args), _vp]),
                       ("cq_norm_residual_a8", [P(cq_norm_args), _vp, _vp, _vp]),
                       ("cq_rope_append", [P(cq_kv_cache), P(cq_rope_args), _vp]),
                       ("cq_attn_paged", [P(cq_kv_cache), P(cq_attn_args), _vp, _i64, _vp]),
                       ("cq_attn_shared_prefix", [P(cq_kv_cache), P(cq_attn_args), _vp, _i64, _vp])):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = args
    L.cq_attn_workspace_bytes.restype = _i64
    L.cq_attn_workspace_bytes.argtypes = [P(cq_kv_cache), P(cq_attn_args)]


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------- norms


def _norm_args(residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out, residual_out):
    torch = _torch()
    rows, width = residual.shape
    assert residual.is_contiguous() and weight.shape == (width,) and weight.is_contiguous()
    dtype, stride = weight.dtype, 0
    if y is not None:
        assert y.shape == residual.shape and y.is_contiguous() and y.dtype == dtype
        if residual_out is None:
            residual_out = torch.empty_like(residual)
        assert residual_out.shape == residual.shape and residual_out.is_contiguous()
        assert residual_out.dtype == residual.dtype
        if post_weight is not None:
            assert post_weight.shape == (width,) and post_weight.is_contiguous() and post_weight.dtype == dtype
        if gate is not None:
            # one gate for all rows, or a row for each
            assert gate.shape[-1] == width and gate.stride(-1) == 1 and gate.dtype == dtype
            if gate.dim() == 2:
                assert gate.shape[0] == rows
                stride = gate.stride(0)
            else:
                assert gate.dim() == 1
    else:
        assert post_weight is None and gate is None and residual_out is None
    if out is not None:
        assert out.shape == residual.shape and out.is_contiguous() and out.dtype == dtype
    args = cq_norm_args(_ptr(y), _ptr(post_weight), _ptr(gate), residual.data_ptr(), weight.data_ptr(),
                        _ptr(residual_out), _ptr(out), stride, rows, width, _dt(dtype), _dt(residual.dtype), alpha,
                        eps, weight_offset)
    return args, residual if y is None else residual_out


def cq_norm_residual(residual, weight, eps, y=None, post_weight=None, gate=None, alpha=1.0, weight_offset=0.0,
                     out=None, residual_out=None, stream=None):
    """r' = residual + alpha * gate * (y or its post norm); h = norm(r') * weight.

    Returns (h, r').  residual [rows, width] in the model dtype or FP32; y,
    weight, post_weight [width] and gate ([width] or [rows, width]) in the model
    dtype.  Without y, r' is the residual itself.  residual_out may be residual,
    out may be y."""
    if out is None:
        out = _torch().empty(residual.shape, dtype=weight.dtype, device=residual.device)
    args, r = _norm_args(residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out, residual_out)
    _check(lib().cq_norm_residual(ctypes.byref(args), _stream_ptr(stream)), "cq_norm_residual")
    return out, r


def cq_norm_residual_a8(residual, weight, eps, y=None, post_weight=None, gate=None, alpha=1.0, weight_offset=0.0,
                        out=None, residual_out=None, x8=None, dx=None, stream=None):
    """cq_norm_residual with h straight to the Dynamic-A8 carriers; returns
    (x8, dx, r').  h itself is written only into a given out."""
    torch = _torch()
    if x8 is None:
        x8 = torch.empty(residual.shape, dtype=torch.int8, device=residual.device)
    if dx is None:
        dx = torch.empty((residual.shape[0],), dtype=torch.float32, device=residual.device)
    assert x8.shape == residual.shape and x8.is_contiguous() and x8.dtype == torch.int8
    assert dx.shape == (residual.shape[0],) and dx.is_contiguous() and dx.dtype == torch.float32
    args, r = _norm_args(residual, weight, eps, y, post_weight, gate, alpha, weight_offset, out, residual_out)
    st = lib().cq_norm_residual_a8(ctypes.byref(args), x8.data_ptr(), dx.data_ptr(), _stream_ptr(stream))
    _check(st, "cq_norm_residual_a8")
    return x8, dx, r


# ---------------------------------------------------------------- the paged cache


def _cache(k_cache, v_cache):
    pages, kv_heads, page, dim = k_cache.shape
    assert v_cache.shape == k_cache.shape and k_cache.is_contiguous() and v_cache.is_contiguous()
    assert v_cache.dtype == k_cache.dtype
    return cq_kv_cache(_dt(k_cache.dtype), kv_heads, dim, page, pages, k_cache.data_ptr(), v_cache.data_ptr())


def _heads_stride(x, dtype, dim):
    """Stride between tokens of x [tokens, heads, dim], whose heads are dense."""
    token, head, one = x.stride()
    assert x.dtype == dtype and x.shape[2] == dim and one == 1 and (head == dim or x.shape[1] == 1)
    # the stride of a single token is never used: any legal one serves
    return token if x.shape[0] > 1 else max(token, x.shape[1] * dim)


def _index(t, shape):
    torch = _torch()
    assert t.dtype == torch.int32 and t.is_contiguous() and t.shape == shape
    return t.data_ptr()


def cq_rope_append(q, k, v, cos, sin, positions, slots, k_cache, v_cache, interleaved=False, q_out=None, stream=None):
    """Rotate q and k by their positions and write k and v into their slots of
    the cache; returns the rotated queries [tokens, heads, dim].

    q, k, v [tokens, heads, dim] may be slices of one fused product; cos, sin
    FP32 [rows, rot / 2], or None for no rotation; positions, slots int32
    [tokens].  q_out may be q."""
    torch = _torch()
    cache = _cache(k_cache, v_cache)
    tokens, heads, dim = q.shape
    assert k.shape == v.shape == (tokens, cache.kv_heads, cache.dim) and dim == cache.dim
    dtype = k_cache.dtype
    if q_out is None:
        q_out = torch.empty((tokens, heads, dim), dtype=dtype, device=q.device)
    assert q_out.shape == q.shape
    rows = rot = 0
    if cos is not None:
        rows, rot = cos.shape[0], 2 * cos.shape[1]
        assert cos.shape == sin.shape and cos.dtype == sin.dtype == torch.float32
        assert cos.is_contiguous() and sin.is_contiguous()
    args = cq_rope_args(q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), _heads_stride(q, dtype, dim),
                        _heads_stride(k, dtype, dim), _heads_stride(v, dtype, dim), _heads_stride(q_out, dtype, dim),
                        _ptr(cos), _ptr(sin), _index(positions, (tokens,)) if rot else None,
                        _index(slots, (tokens,)), tokens, rows, heads, rot, interleaved)
    _check(lib().cq_rope_append(ctypes.byref(cache), ctypes.byref(args), _stream_ptr(stream)), "cq_rope_append")
    return q_out


def _attn(call, where, q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts, max_q, scale, softcap, window, slopes,
          bidir, prefix_table, prefix_len, out, workspace, stream):
    torch = _torch()
    cache = _cache(k_cache, v_cache)
    tokens, heads, dim = q.shape
    batch = kv_lens.shape[0]
    if out is None:
        out = torch.empty((tokens, heads, dim), dtype=q.dtype, device=q.device)
    assert out.shape == q.shape and out.is_contiguous() and out.dtype == q.dtype
    if slopes is not None:
        assert slopes.shape == (heads,) and slopes.dtype == torch.float32 and slopes.is_contiguous()
    args = cq_attn_args(
        q.data_ptr(), out.data_ptr(), _heads_stride(q, k_cache.dtype, cache.dim), tokens, heads, batch,
        None if q_starts is None else _index(q_starts, (batch + 1,)), _index(tables, (batch, tables.shape[1])),
        tables.shape[1], max_q, max_kv, _index(kv_lens, (batch,)), dim**-0.5 if scale is None else scale, softcap,
        window, _ptr(slopes), None if bidir is None else _index(bidir, (batch,)),
        None if prefix_table is None else _index(prefix_table, prefix_table.shape), prefix_len)
    L = lib()
    if workspace is None:
        need = L.cq_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(args))
        if need > 0:
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
    st = getattr(L, call)(ctypes.byref(cache), ctypes.byref(args), _ptr(workspace),
                          0 if workspace is None else workspace.numel() * workspace.element_size(),
                          _stream_ptr(stream))
    _check(st, where)
    return out


def cq_attn_paged(q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts=None, max_q=1, scale=None, softcap=0.0,
                  window=0, slopes=None, bidir=None, out=None, workspace=None, stream=None):
    """Attention of the sequences' newest tokens over the paged cache; returns
    [tokens, heads, dim].

    q [tokens, heads, dim] may be a slice of a fused product; tables int32
    [batch, width], kv_lens int32 [batch]; q_starts int32 [batch + 1], or None
    for one query of every sequence; max_q and max_kv bound the sequences.
    scale defaults to dim ** -0.5.  A workspace given by the caller (uint8,
    cq_attn_workspace_bytes) must not be shared by calls that can overlap."""
    return _attn("cq_attn_paged", "cq_attn_paged", q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts, max_q,
                 scale, softcap, window, slopes, bidir, None, 0, out, workspace, stream)


def cq_attn_shared_prefix(q, k_cache, v_cache, prefix_table, prefix_len, tables, kv_lens, max_kv, q_starts=None,
                          max_q=1, scale=None, softcap=0.0, out=None, workspace=None, stream=None):
    """cq_attn_paged for sequences that all begin with the prefix_len tokens of
    prefix_table (int32), which are read once; tables, kv_lens and max_kv
    describe each one's own tokens behind them."""
    assert prefix_table is None or prefix_len <= prefix_table.numel() * k_cache.shape[2]
    return _attn("cq_attn_shared_prefix", "cq_attn_shared_prefix", q, k_cache, v_cache, tables, kv_lens, max_kv,
                 q_starts, max_q, scale, softcap, 0, None, None, prefix_table, prefix_len, out, workspace, stream)


def cq_attn_workspace_bytes(q, k_cache, v_cache, tables, kv_lens, max_kv, q_starts=None, max_q=1, prefix_len=0):
    """Bytes of workspace that an attention call of these sizes needs."""
    cache = _cache(k_cache, v_cache)
    tokens, heads, dim = q.shape
    table = tables.data_ptr() if prefix_len else None
    args = cq_attn_args(q.data_ptr(), q.data_ptr(), _heads_stride(q, k_cache.dtype, dim), tokens, heads,
                        kv_lens.shape[0], _ptr(q_starts), tables.data_ptr(), tables.shape[1], max_q, max_kv,
                        kv_lens.data_ptr(), 1.0, 0.0, 0, None, None, table, prefix_len)
    return int(lib().cq_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(args)))
