"""The operators of a mixture-of-experts layer beside its packed products
(include/cq_experts.h): routing, 8-bit products dense and of routed experts, the
gated activation, and the sum of the experts' outputs.

Arguments are device tensors; the binding only marshals them.  A call given a
stream runs there, and what it allocates is allocated there; the caller orders it
with the streams that made its arguments and that use its results.
"""
from __future__ import annotations

import ctypes
import struct

from . import CQError, block, lib
from .block import _on, _ptr, _type, _types, _vector

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float

SCORING = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {"silu": 0, "gelu": 1}


class cq_route_args(ctypes.Structure):
    _fields_ = [("logits", _vp), ("bias", _vp), ("live", _vp), ("chosen", _vp), ("weights", _vp), ("plan", _vp),
                ("tokens", _i64), ("stride", _i64), ("dtype", _i32), ("experts", _i32), ("top", _i32),
                ("scoring", _i32), ("groups", _i32), ("kept_groups", _i32), ("group_top", _i32), ("renormalize", _i32),
                ("scale", _f32)]


class cq_w8_args(ctypes.Structure):
    _fields_ = [("x8", _vp), ("dx", _vp), ("w8", _vp), ("dw", _vp), ("bias", _vp), ("y", _vp), ("rows", _i64),
                ("n", _i64), ("k", _i64), ("y_dtype", _i32), ("experts", _i32), ("plan", _vp), ("routes", _i64),
                ("fan", _i32)]


class cq_gated_args(ctypes.Structure):
    _fields_ = [("gate", _vp), ("up", _vp), ("out", _vp), ("rows", _i64), ("width", _i64), ("stride", _i64),
                ("dtype", _i32), ("act", _i32)]


class cq_combine_args(ctypes.Structure):
    _fields_ = [("y", _vp), ("weights", _vp), ("chosen", _vp), ("base", _vp), ("out", _vp), ("tokens", _i64),
                ("width", _i64), ("top", _i32), ("experts", _i32), ("dtype", _i32), ("out_dtype", _i32),
                ("alpha", _f32)]


# The same structures as bytes, packed in one step (as in block.py).
_ROUTE = struct.Struct("@6P2q8if4x")
_W8 = struct.Struct("@6P3q2iPqi4x")
_GATED = struct.Struct("@3P3q2i")
_COMBINE = struct.Struct("@5P2q4if4x")
for _s, _c in ((_ROUTE, cq_route_args), (_W8, cq_w8_args), (_GATED, cq_gated_args), (_COMBINE, cq_combine_args)):
    assert _s.size == ctypes.sizeof(_c), _c


def declare(L):
    """Argument types of the entry points in a loaded library (structures by address)."""
    for name, args in (("cq_route", [_vp, _vp, _i64, _vp]),
                       ("cq_route_plan", [_vp, _i64, _i32, _vp, _vp, _i64, _vp]),
                       ("cq_gemm_w8", [_vp, _vp]),
                       ("cq_gemm_routed_w8", [_vp, _vp]),
                       ("cq_gated", [_vp, _vp]),
                       ("cq_gated_a8", [_vp, _vp, _vp, _vp]),
                       ("cq_combine", [_vp, _vp])):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = args
    L.cq_probe_w8_kernel.restype = _i32
    L.cq_probe_w8_kernel.argtypes = [_vp, _i32, ctypes.POINTER(_i32)]
    for name, args in (("cq_route_workspace_bytes", [_vp]), ("cq_route_plan_workspace_bytes", [_i64, _i32])):
        getattr(L, name).restype = _i64
        getattr(L, name).argtypes = args


torch = None  # imported with the first call, as by the package
_device = _raw_stream = None


def _torch():
    global torch, _device, _raw_stream
    if torch is None:
        t = block._torch()
        # current device, and handle of its current stream: a tenth of a microsecond each
        _device, _raw_stream = t._C._cuda_getDevice, t._C._cuda_getCurrentRawStream
        torch = t
    return torch


def _begin(*tensors):
    """The stream of the call, that of the current device, on which all tensors lie."""
    device = _device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"a tensor on {t.device} in a call on cuda:{device}")
    return _raw_stream(device)


def _check(st, where):
    if st:
        raise CQError(st, where)


def _out(t, shape, dtype, like):
    """A given output of this shape and type, or a new one."""
    if t is None:
        return like.new_empty(shape, dtype=dtype)
    assert t.dtype == dtype and t.shape == shape and t.is_contiguous()
    return t


def _room(workspace, need, like):
    """(workspace, its bytes): the caller's, or a new one of the bytes that are needed."""
    if workspace is not None:
        assert workspace.is_contiguous()
        return workspace, workspace.numel() * workspace.element_size()
    return like.new_empty((need,), dtype=torch.uint8) if need > 0 else None, need


# ---------------------------------------------------------------- routing


def cq_route(logits, top, scoring="softmax", bias=None, groups=1, kept_groups=1, group_top=1, renormalize=True,
             scale=1.0, live=None, chosen=None, weights=None, plan=None, workspace=None, stream=None):
    """The experts of every token; returns (chosen int32 [tokens, top], weights
    FP32 [tokens, top], plan int32 [experts + 1 + tokens * top]).

    logits [tokens, experts] in BF16, FP16 or FP32, rows of any stride; bias FP32
    [experts] is added to the scores for the choice alone; live int32 [1]: tokens
    from there on have no experts.  The plan is that of cq_route_plan.  A workspace
    given by the caller must not be shared by calls that can overlap."""
    _torch()
    if stream is not None:
        return _on(stream, cq_route, logits, top, scoring, bias, groups, kept_groups, group_top, renormalize, scale,
                   live, chosen, weights, plan, workspace)
    on = _begin(logits, bias, live, chosen, weights, plan, workspace)
    tokens, experts = logits.shape
    assert logits.stride(1) == 1 or experts == 1
    int32 = torch.int32
    chosen = _out(chosen, (tokens, top), int32, logits)
    weights = _out(weights, (tokens, top), torch.float32, logits)
    plan = _out(plan, (experts + 1 + tokens * top,), int32, logits)
    args = _ROUTE.pack(logits.data_ptr(), 0 if bias is None else _vector(bias, experts, torch.float32),
                       0 if live is None else _vector(live, 1, int32), chosen.data_ptr(), weights.data_ptr(),
                       plan.data_ptr(), tokens, logits.stride(0) if tokens > 1 else experts, _type(logits), experts,
                       top, SCORING[scoring], groups, kept_groups, group_top, renormalize, scale)
    L = lib()
    workspace, size = _room(workspace, L.cq_route_workspace_bytes(args) if workspace is None else 0, logits)
    _check(L.cq_route(args, _ptr(workspace), size, on), "cq_route")
    return chosen, weights, plan


def cq_route_plan(chosen, experts, plan=None, workspace=None, stream=None):
    """The routes of a map (int32, any shape; route r is its r-th element) in the
    order of their experts: int32 [experts + 1 + routes], offsets and then routes."""
    _torch()
    if stream is not None:
        return _on(stream, cq_route_plan, chosen, experts, plan, workspace)
    on = _begin(chosen, plan, workspace)
    assert chosen.dtype == torch.int32 and chosen.is_contiguous()
    routes = chosen.numel()
    plan = _out(plan, (experts + 1 + routes,), torch.int32, chosen)
    L = lib()
    workspace, size = _room(workspace, L.cq_route_plan_workspace_bytes(routes, experts) if workspace is None else 0,
                            chosen)
    _check(L.cq_route_plan(chosen.data_ptr(), routes, experts, plan.data_ptr(), _ptr(workspace), size, on),
           "cq_route_plan")
    return plan


# ---------------------------------------------------------------- products of 8-bit integers


def _dense8(t):
    assert t.dtype == torch.int8 and t.is_contiguous()
    return t.data_ptr()


def cq_gemm_w8(x8, dx, w8, dw, bias=None, y_dtype=None, out=None, stream=None):
    """y = (x8 w8^T) dx dw + bias; returns [rows, n] in y_dtype (BF16 by default).

    x8 int8 [rows, k] and dx FP32 [rows] as of cq_quantize_act_a8; w8 int8 [n, k]
    with a scale for each channel, dw FP32 [n]; bias [n] in y_dtype."""
    _torch()
    if stream is not None:
        return _on(stream, cq_gemm_w8, x8, dx, w8, dw, bias, y_dtype, out)
    on = _begin(x8, dx, w8, dw, bias, out)
    rows, k = x8.shape
    n = w8.shape[0]
    assert w8.shape == (n, k)
    if y_dtype is None:
        y_dtype = torch.bfloat16 if out is None else out.dtype
    out = _out(out, (rows, n), y_dtype, x8)
    args = _W8.pack(_dense8(x8), _vector(dx, rows, torch.float32), _dense8(w8), _vector(dw, n, torch.float32),
                    0 if bias is None else _vector(bias, n, y_dtype), out.data_ptr(), rows, n, k, _type(out), 0, 0, 0,
                    0)
    _check(lib().cq_gemm_w8(args, on), "cq_gemm_w8")
    return out


def cq_gemm_routed_w8(x8, dx, w8, dw, plan, fan=1, bias=None, y_dtype=None, out=None, stream=None):
    """cq_gemm_w8 of routed experts; returns [routes, n], a row for each route.

    w8 int8 [experts, n, k], dw FP32 [experts, n], bias [experts, n]; plan of
    cq_route or cq_route_plan.  Route r takes row r // fan of x8: fan is the routes
    of a token where x8 has a row for each token, 1 where it has one for each
    route.  Rows of routes without an expert are not written."""
    _torch()
    if stream is not None:
        return _on(stream, cq_gemm_routed_w8, x8, dx, w8, dw, plan, fan, bias, y_dtype, out)
    on = _begin(x8, dx, w8, dw, plan, bias, out)
    rows, k = x8.shape
    experts, n, _ = w8.shape
    assert w8.shape[2] == k and dw.shape == (experts, n) and dw.dtype == torch.float32 and dw.is_contiguous()
    routes = plan.numel() - experts - 1
    if y_dtype is None:
        y_dtype = torch.bfloat16 if out is None else out.dtype
    out = _out(out, (routes, n), y_dtype, x8)
    if bias is not None:
        assert bias.shape == dw.shape and bias.dtype == y_dtype and bias.is_contiguous()
    args = _W8.pack(_dense8(x8), _vector(dx, rows, torch.float32), _dense8(w8), dw.data_ptr(), _ptr(bias),
                    out.data_ptr(), rows, n, k, _type(out), experts, _vector(plan, plan.numel(), torch.int32), routes,
                    fan)
    _check(lib().cq_gemm_routed_w8(args, on), "cq_gemm_routed_w8")
    return out


W8_KERNELS = (None, "few", "rows", "tiles", "tiles far")


def cq_probe_w8_kernel(rows, n, k, experts=0, routes=0, fan=1):
    """Kernel that a product of these sizes takes, routed if it has experts: (name, rows
    and channels of a workgroup, stages in flight), or None where it is refused."""
    at, tile = 4096, (_i32 * 3)()  # any aligned address: none is read
    args = _W8.pack(at, at, at, at, 0, at, rows, n, k, 0, experts, at if experts else 0, routes, fan if experts else 0)
    kernel = lib().cq_probe_w8_kernel(args, int(experts > 0), tile)
    return (W8_KERNELS[kernel], *tile) if kernel else None


# ---------------------------------------------------------------- between the products and behind them


def _gated_args(gate, up, act, out):
    shape, strides = gate.shape, gate.stride()
    rows, width = shape
    assert up.shape == shape and up.dtype == gate.dtype
    # the stride of a single row is never used: any legal one serves
    stride = strides[0] if rows > 1 else width
    assert strides[1] == 1 and (up.stride() == strides or rows == 1 and up.stride(1) == 1)
    return _GATED.pack(gate.data_ptr(), up.data_ptr(), 0 if out is None else out.data_ptr(), rows, width, stride,
                       _type(gate), ACTIVATIONS[act])


def cq_gated(gate, up, act="silu", out=None, stream=None):
    """act(gate) * up; returns [rows, width].  gate and up [rows, width] may be the
    halves of one product's output; act is silu or gelu (by tanh)."""
    _torch()
    if stream is not None:
        return _on(stream, cq_gated, gate, up, act, out)
    on = _begin(gate, up, out)
    # an empty_like is dense here, and takes two thirds of a new_empty's time
    out = torch.empty_like(gate) if out is None else _out(out, gate.shape, gate.dtype, gate)
    _check(lib().cq_gated(_gated_args(gate, up, act, out), on), "cq_gated")
    return out


def cq_gated_a8(gate, up, act="silu", out=None, x8=None, dx=None, stream=None):
    """cq_gated straight to the Dynamic-A8 carriers; returns (x8, dx).  The
    activation itself is written only into a given out."""
    _torch()
    if stream is not None:
        return _on(stream, cq_gated_a8, gate, up, act, out, x8, dx)
    on = _begin(gate, up, out, x8, dx)
    if out is not None:
        _out(out, gate.shape, gate.dtype, gate)
    x8 = _out(x8, gate.shape, torch.int8, gate)
    dx = _out(dx, gate.shape[:1], torch.float32, gate)
    _check(lib().cq_gated_a8(_gated_args(gate, up, act, out), x8.data_ptr(), dx.data_ptr(), on),
           "cq_gated_a8")
    return x8, dx


def cq_combine(y, weights, chosen, experts, base=None, alpha=1.0, out=None, stream=None):
    """base + alpha * sum over a token's routes of weight * y; returns [tokens, width].

    y [tokens * top, width], weights FP32 and chosen int32 [tokens, top] of cq_route;
    routes whose expert is outside 0 .. experts - 1 have no part.  base [tokens,
    width] (a shared expert's output, or the stream) in the type of y or in FP32;
    the result has its type.  out may be base."""
    _torch()
    if stream is not None:
        return _on(stream, cq_combine, y, weights, chosen, experts, base, alpha, out)
    on = _begin(y, weights, chosen, base, out)
    tokens, top = chosen.shape
    routes, width = y.shape
    assert routes == tokens * top and y.is_contiguous()
    assert chosen.dtype == torch.int32 and chosen.is_contiguous()
    assert weights.dtype == torch.float32 and weights.shape == chosen.shape and weights.is_contiguous()
    if base is not None:
        assert base.shape == (tokens, width) and base.is_contiguous()
        dtype = base.dtype
        out = torch.empty_like(base) if out is None else _out(out, (tokens, width), dtype, y)
    else:
        dtype = y.dtype if out is None else out.dtype
        out = _out(out, (tokens, width), dtype, y)
    args = _COMBINE.pack(y.data_ptr(), weights.data_ptr(), chosen.data_ptr(), _ptr(base), out.data_ptr(), tokens, width,
                         top, experts, _type(y), _types[dtype], alpha)
    _check(lib().cq_combine(args, on), "cq_combine")
    return out
