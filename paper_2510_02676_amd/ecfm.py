"""Thin Python binding of the products of many rows and of a mixture of experts (``include/ecfm.h``).

Argument marshalling only; every step runs inside ``libecf8.so`` (importing this module fails loudly when the library is
not built).  ``Weights`` holds the C structure of one matrix, or of all experts' matrices, and keeps the tensors alive; it is made once.
``Routes`` holds what ``ecfm_route`` writes and its workspace; a loop keeps one.  Streams, allocated results and devices are handled as in ``ecfa``: a
call on another stream makes what it allocates of that stream's memory, and all tensors of a call are on that stream's device, or it
is refused (``E_ARG``).
"""
import ctypes

import torch

from . import ecf8 as _e
from .ecfa import _BYTES, _DTYPE, _bad, _empty, _stream_ptr

_lib = _e._lib
_U32 = (1 << 32) - 1
_vp, _u64, _u32, _i64, _f32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int64, ctypes.c_float


class _Weights(ctypes.Structure):
    _fields_ = [("d", _vp), ("d_scale", _vp), ("row_stride", _i64), ("expert_stride", _i64), ("rows", _u32), ("cols", _u32), ("experts", _u32),
                ("reserved", _u32)]


class _X(ctypes.Structure):
    _fields_ = [("d", _vp), ("d_scale", _vp), ("row_stride", _i64), ("rows", _u32), ("scale_cols", _u32)]


class _Y(ctypes.Structure):
    _fields_ = [("d", _vp), ("row_stride", _i64), ("rows", _u32), ("dtype", _u32)]


class _RouteOpts(ctypes.Structure):
    _fields_ = [("d_logits", _vp), ("d_bias", _vp), ("logit_stride", _i64), ("n_tokens", _u32), ("experts", _u32), ("top", _u32), ("dtype", _u32),
                ("sigmoid", _u32), ("normalise", _u32), ("groups", _u32), ("top_groups", _u32), ("scale", _f32), ("reserved", _u32)]


_P = ctypes.POINTER
_lib.ecfm_gemm.argtypes = [_P(_Weights), _P(_X), _P(_Y), _vp]
_lib.ecfm_gemm_experts.argtypes = [_P(_Weights), _vp, _P(_X), _vp, _P(_Y), _vp]
_lib.ecfm_route_workspace_bytes.argtypes = [_u32, _u32, _u32]
_lib.ecfm_route_workspace_bytes.restype = _u64
_lib.ecfm_route.argtypes = [_P(_RouteOpts), _vp, _vp, _vp, _vp, _vp, _vp, _u64, _vp]
_lib.ecfm_gate.argtypes = [_vp, _vp, _u32, _u64, _u64, _i64, _i64, _u32, _vp, _vp, _vp]
_lib.ecfm_combine.argtypes = [_P(_Y), _vp, _vp, _u32, _u32, _u32, _P(_Y), _P(_Y), _vp]

_gemm, _gemm_experts, _route, _gate, _combine = _lib.ecfm_gemm, _lib.ecfm_gemm_experts, _lib.ecfm_route, _lib.ecfm_gate, _lib.ecfm_combine


def _dense(fn, t, dtype, shape, on):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != on:
        raise _bad(fn)
    return t.data_ptr()


def _matrix(fn, y, rows, cols, on):
    """A (rows, cols) tensor of fp32 or BF16 as the C structure: any distance between rows, columns next to each other."""
    stride, dtype = y.stride(), _DTYPE.get(y.dtype)
    if y.shape != (rows, cols) or dtype is None or (stride[1] != 1 and cols > 1) or y.get_device() != on or rows > _U32:
        raise _bad(fn)
    return _Y(y.data_ptr(), stride[0], rows, dtype)


class Weights:
    """Decoded weights of a product, (rows, cols), or of several experts, (experts, rows, cols): E4M3 (``torch.float8_e4m3fn``, or uint8 holding
    its bytes), columns next to each other, any other strides; scale fp32 (rows / 128, cols / 128) rounded up, with the experts in front, or None."""

    def __init__(self, w, scale=None):
        if w.dim() not in (2, 3) or w.dtype not in _BYTES or (w.shape[-1] > 1 and w.stride(-1) != 1) or 0 in w.shape or any(n >= 1 << 32 for n in w.shape):
            raise _bad("Weights")
        rows, cols = w.shape[-2:]
        self.w, self.scale, self.on, self.device = w, scale, w.get_device(), w.device
        self.experts, self.rows, self.cols = (w.shape[0] if w.dim() == 3 else 1), rows, cols
        self.blocks = -(-cols // 128)
        self.c = _Weights(w.data_ptr(), None if scale is None else _dense("Weights", scale, torch.float32, (*w.shape[:-2], -(-rows // 128), self.blocks), self.on),
                          w.stride(-2), w.stride(0) if w.dim() == 3 else 0, rows, cols, self.experts, 0)


def _x(fn, weights, x, scale):
    """X (rows, cols) of E4M3 and its scales (rows,), (rows, 1) or (rows, cols / 128 rounded up), or None, as the C structure."""
    shape, stride, on = x.shape, x.stride(), weights.on
    if len(shape) != 2 or shape[1] != weights.cols or x.dtype not in _BYTES or (shape[1] > 1 and stride[1] != 1) or x.get_device() != on or shape[0] >= 1 << 32:
        raise _bad(fn)
    if scale is None:
        return _X(x.data_ptr(), None, stride[0], shape[0], 0)
    per = scale.shape[1] if scale.dim() == 2 else 1
    if (per != 1 and per != weights.blocks) or scale.dim() not in (1, 2):
        raise _bad(fn)
    return _X(x.data_ptr(), _dense(fn, scale, torch.float32, (shape[0], per) if scale.dim() == 2 else (shape[0],), on), stride[0], shape[0], per)


def ecfm_gemm(weights, x, x_scale=None, y=None, dtype=torch.bfloat16, stream=None):
    """Y = X W^T: x (m, cols) E4M3 with x_scale (m,) or (m, cols / 128 rounded up) fp32 or None; y (m, rows) BF16 or fp32, allocated in `dtype` if absent."""
    if weights.w.dim() != 2:
        raise _bad("ecfm_gemm")
    at = _stream_ptr("ecfm_gemm", weights.on, stream)
    cx = _x("ecfm_gemm", weights, x, x_scale)
    if y is None:
        if dtype not in _DTYPE:
            raise _bad("ecfm_gemm")
        y = _empty((cx.rows, weights.rows), dtype, weights.device, stream)
    rc = _gemm(weights.c, cx, _matrix("ecfm_gemm", y, cx.rows, weights.rows, weights.on), at)
    if rc:
        _e._check("ecfm_gemm", rc)
    return y


def ecfm_gemm_experts(weights, starts, x, x_scale=None, rows=None, y=None, dtype=torch.bfloat16, stream=None):
    """Row p of the result, starts[e] <= p < starts[e + 1], is row rows[p] of x (row p if rows is None) times expert e's weights.  weights: of a
    (experts, rows, cols) tensor; starts (experts + 1,) and rows int32.  Rows that belong to no expert are not written: in a result that is
    allocated here they are undefined."""
    on = weights.on
    if weights.w.dim() != 3:
        raise _bad("ecfm_gemm_experts")
    at = _stream_ptr("ecfm_gemm_experts", on, stream)
    cx = _x("ecfm_gemm_experts", weights, x, x_scale)
    begin = _dense("ecfm_gemm_experts", starts, torch.int32, (weights.experts + 1,), on)
    n = cx.rows if rows is None else rows.shape[0] if rows.dim() == 1 else -1
    which = None if rows is None else _dense("ecfm_gemm_experts", rows, torch.int32, (n,), on)
    if y is None:
        if dtype not in _DTYPE:
            raise _bad("ecfm_gemm_experts")
        y = _empty((n, weights.rows), dtype, weights.device, stream)
    rc = _gemm_experts(weights.c, begin, cx, which, _matrix("ecfm_gemm_experts", y, n, weights.rows, on), at)
    if rc:
        _e._check("ecfm_gemm_experts", rc)
    return y


class Routes:
    """Where the tokens of a step go, as ``ecfm_route`` leaves it: ids and weights (tokens, top), starts (experts + 1,), rows (tokens * top,) and
    place (tokens, top), all int32 but the fp32 weights."""

    def __init__(self, tokens, top, experts, device="cuda", stream=None):
        if not (0 <= tokens <= 1 << 22 and 1 <= top <= 32 and top <= experts <= 1024):
            raise _bad("Routes")
        new = lambda *shape, dtype=torch.int32: _empty(shape, dtype, device, stream)  # noqa: E731
        self.tokens, self.top, self.experts = tokens, top, experts
        self.ids, self.weights, self.starts = new(tokens, top), new(tokens, top, dtype=torch.float32), new(experts + 1)
        self.rows, self.place = new(tokens * top), new(tokens, top)
        n = int(_lib.ecfm_route_workspace_bytes(tokens, experts, top))
        self.workspace = new(n, dtype=torch.uint8) if n else None
        self.on = self.ids.get_device()
        self.at = (self.ids.data_ptr(), self.weights.data_ptr(), self.starts.data_ptr(), self.rows.data_ptr(), self.place.data_ptr(),
                   self.workspace.data_ptr() if n else None, n)


def ecfm_route(logits, top, sigmoid=False, bias=None, groups=1, top_groups=1, normalise=True, scale=1.0, routes=None, stream=None):
    """The `top` experts of each row of logits (tokens, experts), fp32 or BF16, and the pairs sorted by expert: a ``Routes``, the given one or a
    new one.  bias (experts,) fp32."""
    shape, stride, dtype = logits.shape, logits.stride(), _DTYPE.get(logits.dtype)
    if len(shape) != 2 or dtype is None or (shape[1] > 1 and stride[1] != 1) or any(not 0 <= v < 1 << 32 for v in (top, groups, top_groups)):
        raise _bad("ecfm_route")
    on = logits.get_device()
    at = _stream_ptr("ecfm_route", on, stream)
    if routes is None:
        routes = Routes(shape[0], top, shape[1], logits.device, stream)
    elif routes.on != on or (routes.tokens, routes.experts) != tuple(shape) or routes.top != top:
        raise _bad("ecfm_route")
    opts = _RouteOpts(logits.data_ptr(), None if bias is None else _dense("ecfm_route", bias, torch.float32, (shape[1],), on), stride[0], shape[0], shape[1], top,
                      dtype, bool(sigmoid), bool(normalise), groups, top_groups, scale, 0)
    rc = _route(opts, *routes.at, at)
    if rc:
        _e._check("ecfm_route", rc)
    return routes


def ecfm_gate(g, u, group=0, q=None, scale=None, stream=None):
    """silu(g) * u, (rows, cols) fp32 or BF16 each, rows of any stride, to (E4M3 (rows, cols), fp32 scales (rows,) or with group = 128 (rows, cols /
    128)); the result is a ``torch.float8_e4m3fn`` tensor unless q is given (uint8 or float8_e4m3fn, dense)."""
    shape, dtype, on = g.shape, _DTYPE.get(g.dtype), g.get_device()
    if len(shape) != 2 or dtype is None or u.shape != shape or u.dtype != g.dtype or u.get_device() != on or group not in (0, 128):
        raise _bad("ecfm_gate")
    at = _stream_ptr("ecfm_gate", on, stream)
    rows, cols = shape
    g_stride, u_stride = g.stride(), u.stride()
    if cols > 1 and (g_stride[1] != 1 or u_stride[1] != 1):
        raise _bad("ecfm_gate")
    want = (rows, cols // 128) if group else (rows,)
    if q is None:
        q = _empty((rows, cols), torch.float8_e4m3fn, g.device, stream)
    if scale is None:
        scale = _empty(want, torch.float32, g.device, stream)
    if q.dtype not in _BYTES or q.shape != shape or not q.is_contiguous() or q.get_device() != on:
        raise _bad("ecfm_gate")
    rc = _gate(g.data_ptr(), u.data_ptr(), dtype, rows, cols, g_stride[0], u_stride[0], group, q.data_ptr(), _dense("ecfm_gate", scale, torch.float32, want, on), at)
    if rc:
        _e._check("ecfm_gate", rc)
    return q, scale


def ecfm_combine(y, place, weights, add=None, out=None, dtype=torch.bfloat16, stream=None):
    """out[t] = add[t] + sum over j of weights[t][j] * y[place[t][j]]: y (rows, cols), add and out (tokens, cols) BF16 or fp32 (out allocated in
    `dtype` if absent, and may be add), place (tokens, top) int32, weights (tokens, top) fp32."""
    on = y.get_device()
    shape, pairs = y.shape, place.shape
    if len(shape) != 2 or len(pairs) != 2:
        raise _bad("ecfm_combine")
    at = _stream_ptr("ecfm_combine", on, stream)
    (rows, cols), (tokens, top) = shape, pairs
    if out is None:
        if dtype not in _DTYPE:
            raise _bad("ecfm_combine")
        out = _empty((tokens, cols), dtype, y.device, stream)
    if tokens > _U32 or top > _U32 or cols > _U32:
        raise _bad("ecfm_combine")
    rc = _combine(_matrix("ecfm_combine", y, rows, cols, on), _dense("ecfm_combine", place, torch.int32, pairs, on),
                  _dense("ecfm_combine", weights, torch.float32, pairs, on), tokens, top, cols,
                  None if add is None else _matrix("ecfm_combine", add, tokens, cols, on), _matrix("ecfm_combine", out, tokens, cols, on), at)
    if rc:
        _e._check("ecfm_combine", rc)
    return out
