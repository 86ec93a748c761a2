"""Thin Python binding of the attention calls (``include/ecfa.h``): what lies between a layer's compressed projections.

Argument marshalling only; every step runs inside ``libecf8.so`` (importing this module fails loudly when the library is
not built).  The objects here hold the C structures and keep the tensors they point to alive: a ``Cache`` and a ``Batch`` are
made once and used by every layer's and every step's calls; the tensors inside them may be rewritten in place.

A call on another stream than the current one (`stream`) makes what it allocates of that stream's memory; the caller orders that stream
behind what wrote the call's inputs, and whatever reads the results behind that stream.  All tensors of a call are on one device, that of its
stream, or it is refused (``E_ARG``).
"""
import ctypes

import torch

from . import ecf8 as _e

_lib = _e._lib
F32, BF16, E4M3 = 1, 2, 3
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_RAMP = 0, 1, 2, 3
_vp, _u64, _u32, _i64, _f32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int64, ctypes.c_float


class _Rows(ctypes.Structure):
    _fields_ = [("d", _vp), ("token_stride", _i64), ("head_stride", _i64), ("heads", _u32), ("dtype", _u32)]


class _Cache(ctypes.Structure):
    _fields_ = [("d_k", _vp), ("d_v", _vp), ("d_k_scale", _vp), ("d_v_scale", _vp), ("k_stride", _i64 * 3), ("v_stride", _i64 * 3),
                ("n_pages", _u32), ("page_size", _u32), ("kv_heads", _u32), ("head_dim", _u32), ("dtype", _u32), ("reserved", _u32)]


class _Batch(ctypes.Structure):
    _fields_ = [("d_page_table", _vp), ("d_kv_len", _vp), ("d_q_start", _vp), ("table_stride", _i64), ("table_width", _u32),
                ("n_seqs", _u32), ("n_tokens", _u32), ("max_q", _u32), ("max_kv", _u32), ("reserved", _u32)]


class _Rope(ctypes.Structure):
    _fields_ = [("d_freq", _vp), ("d_pos", _vp), ("rot_dim", _u32), ("interleaved", _u32), ("scale", _f32), ("reserved", _u32)]


class _AttendOpts(ctypes.Structure):
    _fields_ = [("scale", _f32), ("softcap", _f32), ("d_slopes", _vp), ("d_prefix_len", _vp), ("causal", _u32), ("window", _u32)]


_P = ctypes.POINTER
_lib.ecfa_rope_freq.argtypes = [_u32, ctypes.c_double, _u32, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double, _P(_u64), _P(_f32)]
_lib.ecfa_append.argtypes = [_P(_Cache), _P(_Batch), _P(_Rope), _P(_Rows), _P(_Rows), _P(_Rows), _P(_Rows), _vp]
_lib.ecfa_attend_workspace_bytes.argtypes = [_P(_Cache), _P(_Batch), _u32]
_lib.ecfa_attend_workspace_bytes.restype = _u64
_lib.ecfa_attend.argtypes = [_P(_Cache), _P(_Batch), _P(_AttendOpts), _P(_Rows), _P(_Rows), _vp, _u64, _vp]
_lib.ecfa_quant.argtypes = [_vp, _u32, _u64, _u64, _i64, _u32, _vp, _vp, _vp]

_append, _attend, _quant = _lib.ecfa_append, _lib.ecfa_attend, _lib.ecfa_quant

_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}
_BYTES = (torch.float8_e4m3fn, torch.uint8)


def _bad(fn):
    return _e.Ecf8Error(fn, _e.E_ARG)


def _stream_ptr(fn, on, stream):
    """The stream's handle, for tensors on the device of number `on` (-1, the host, is nobody's): it has to be one of that device's."""
    if stream is not None:
        if stream.device_index != on:
            raise _bad(fn)
    elif on < 0 or _e._device_now() != on:
        raise _bad(fn)
    elif _e._raw_stream is not None:
        return _e._raw_stream(on)
    return _e._stream_ptr(stream)


def _rows(fn, x, n_tokens, heads, dim, on):
    """A (tokens, heads, dim) tensor as the C structure: any strides, elements of a head next to each other."""
    shape, stride, dtype = x.shape, x.stride(), _DTYPE.get(x.dtype)
    if len(shape) != 3 or shape[0] != n_tokens or shape[2] != dim or (heads and shape[1] != heads) or dtype is None or stride[2] != 1 or x.get_device() != on:
        raise _bad(fn)
    return _Rows(x.data_ptr(), stride[0], stride[1], shape[1], dtype)


def _i32(fn, t, shape, on):
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != on:
        raise _bad(fn)
    return t.data_ptr()


def _scale_ptr(t, heads, on):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (heads,) or not t.is_contiguous() or t.get_device() != on:
        raise _bad("Cache")
    return t.data_ptr()


def _empty(shape, dtype, device, stream):
    """Memory for a call on `stream` (None: the current one).  It comes from that stream's own: a block of the current stream's may still be in use by
    kernels queued there, which nothing orders `stream` behind.  The current stream is noted as a user of it, for the program that gets it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        x = torch.empty(shape, dtype=dtype, device=device)
    x.record_stream(torch.cuda.current_stream(device))
    return x


class Cache:
    """A pool of pages: k and v are (pages, page_size, kv_heads, head_dim) tensors of BF16 or E4M3 (``torch.float8_e4m3fn``, or uint8
    holding its bytes), of any strides over the first three dimensions; k_scale and v_scale (kv_heads,) fp32 or None."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride(3) != 1 or v.stride(3) != 1 or k.get_device() != v.get_device():
            raise _bad("Cache")
        if k.dtype == torch.bfloat16:
            dtype = BF16
        elif k.dtype in _BYTES:
            dtype = E4M3
        else:
            raise _bad("Cache")
        pages, page, heads, dim = k.shape
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.on = k.get_device()
        self.c = _Cache(k.data_ptr(), v.data_ptr(), _scale_ptr(k_scale, heads, self.on), _scale_ptr(v_scale, heads, self.on), (_i64 * 3)(*k.stride()[:3]),
                        (_i64 * 3)(*v.stride()[:3]), pages, page, heads, dim, dtype, 0)
        self.kv_heads, self.head_dim, self.device, self.scale = heads, dim, k.device, dim ** -0.5 if dim else 1.0


class Batch:
    """One step of a serving loop, over tensors that the loop rewrites in place: page_table (seqs, width) int32, kv_len (seqs,) int32
    with the new tokens counted, q_start (seqs + 1,) int32 (None: one new token each).  n_tokens: rows of q, k, v and out (default with
    q_start None: seqs).  max_q, max_kv: the most new tokens and keys of a sequence, hints for how the work is split."""

    def __init__(self, page_table, kv_len, q_start=None, n_tokens=None, max_q=0, max_kv=0):
        if page_table.dim() != 2 or page_table.dtype != torch.int32 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise _bad("Batch")
        seqs, width = page_table.shape
        if n_tokens is None:
            if q_start is not None:
                raise _bad("Batch")
            n_tokens = seqs
        if any(not 0 <= x < 1 << 32 for x in (n_tokens, max_q, max_kv)):
            raise _bad("Batch")
        self.page_table, self.kv_len, self.q_start = page_table, kv_len, q_start
        self.n_tokens = n_tokens
        self.on = page_table.get_device()
        self.c = _Batch(page_table.data_ptr(), _i32("Batch", kv_len, (seqs,), self.on), None if q_start is None else _i32("Batch", q_start, (seqs + 1,), self.on),
                        page_table.stride(0), width, seqs, n_tokens, max_q, max_kv, 0)


def rope_freq(rot_dim, base=10000.0, kind=ROPE_PLAIN, factor=1.0, original_len=0.0, beta_fast=32.0, beta_slow=1.0, device="cuda"):
    """(frequencies as int64 bit patterns on the device, scale) of ``ecfa_rope_freq``: what a ``Rope`` takes."""
    if not 0 < rot_dim < 1 << 32:                                # (as 32 bits it would be another number, of more frequencies than there is room for)
        raise _bad("ecfa_rope_freq")
    freq, scale = (_u64 * max(1, rot_dim // 2))(), _f32()
    _e._check("ecfa_rope_freq", _lib.ecfa_rope_freq(rot_dim, base, kind, factor, original_len, beta_fast, beta_slow, freq, ctypes.byref(scale)))
    return torch.tensor([int(f) for f in freq], dtype=torch.int64).to(device), float(scale.value)


class Rope:
    """The rotation: freq (rot_dim / 2,) int64 as ``rope_freq`` gives it; pos (n_tokens,) int32 where positions are not the
    places in the cache."""

    def __init__(self, freq, interleaved=False, scale=1.0, pos=None):
        if freq.dim() != 1 or freq.dtype != torch.int64 or not freq.is_contiguous():
            raise _bad("Rope")
        self.freq, self.pos = freq, pos
        self.on = freq.get_device()
        self.c = _Rope(freq.data_ptr(), None if pos is None else _i32("Rope", pos, pos.shape, self.on), 2 * freq.numel(), int(interleaved), scale, 0)


def ecfa_append(cache, batch, k=None, v=None, q=None, q_out=None, rope=None, stream=None):
    """k turned and v into the cache, q turned into q_out (allocated if absent), which is returned.  k, v: (n_tokens, kv_heads,
    head_dim), q: (n_tokens, heads, head_dim), all fp32 or all BF16."""
    n, dim, on = batch.n_tokens, cache.head_dim, cache.on
    if batch.on != on or (rope is not None and (rope.on != on or (rope.pos is not None and rope.pos.numel() != n))):
        raise _bad("ecfa_append")
    at = _stream_ptr("ecfa_append", on, stream)
    rk = None if k is None else _rows("ecfa_append", k, n, cache.kv_heads, dim, on)
    rv = None if v is None else _rows("ecfa_append", v, n, cache.kv_heads, dim, on)
    rq = ro = None
    if q is not None:
        rq = _rows("ecfa_append", q, n, 0, dim, on)
        if q_out is None:
            q_out = _empty(q.shape, torch.bfloat16, q.device, stream)
        ro = _rows("ecfa_append", q_out, n, q.shape[1], dim, on)
    elif q_out is not None:
        raise _bad("ecfa_append")
    rc = _append(cache.c, batch.c, None if rope is None else rope.c, rq, rk, rv, ro, at)
    if rc:
        _e._check("ecfa_append", rc)
    return q_out


def attend_workspace(cache, batch, heads, stream=None):
    """A workspace for ``ecfa_attend`` with `heads` query heads on this batch (a uint8 tensor, for one call at a time, on `stream`), or None if the
    calls need none."""
    n = int(_lib.ecfa_attend_workspace_bytes(cache.c, batch.c, heads))
    return _empty(n, torch.uint8, cache.device, stream) if n else None


def _opts(fn, cache, batch, heads, scale=None, causal=True, window=0, softcap=0.0, slopes=None, prefix=None):
    """The options of ``ecfa_attend`` as the C structure."""
    if not 0 <= window < 1 << 32:
        raise _bad(fn)
    if slopes is not None and (slopes.dtype != torch.float32 or slopes.shape != (heads,) or not slopes.is_contiguous() or slopes.get_device() != cache.on):
        raise _bad(fn)
    return _AttendOpts(cache.scale if scale is None else scale, softcap, None if slopes is None else slopes.data_ptr(),
                       None if prefix is None else _i32(fn, prefix, batch.kv_len.shape, cache.on), int(causal), window)


def check_layer(fn, cache, batch, heads, rope=None, **options):
    """Raises what ``ecfa_append`` and ``ecfa_attend`` would for these and rows of `heads` query heads, and launches nothing: for programs that build a
    layer before its first step.  The calls are made for a batch of no tokens."""
    if batch.on != cache.on or cache.on < 0 or (rope is not None and (rope.on != cache.on or (rope.pos is not None and rope.pos.numel() != batch.n_tokens))):
        raise _bad(fn)
    opts = _opts(fn, cache, batch, heads, **options)
    none = Batch(batch.page_table[:0], batch.kv_len[:0])
    q, k = (_Rows(None, 0, 0, n, BF16) for n in (heads, cache.kv_heads))
    _e._check(fn, _append(cache.c, none.c, None if rope is None else rope.c, q, k, k, q, None))
    _e._check(fn, _attend(cache.c, none.c, opts, q, q, None, 0, None))


def ecfa_attend(cache, batch, q, scale=None, causal=True, window=0, softcap=0.0, slopes=None, prefix=None, out=None, workspace=None, stream=None):
    """Attention of the batch's new tokens over the cache; q and the result (n_tokens, heads, head_dim) BF16.  scale defaults to
    head_dim^-0.5; slopes (heads,) fp32; prefix (seqs,) int32.  Without a workspace one is allocated for the call where it needs it."""
    n, dim, on = batch.n_tokens, cache.head_dim, cache.on
    if batch.on != on:
        raise _bad("ecfa_attend")
    at = _stream_ptr("ecfa_attend", on, stream)
    rq = _rows("ecfa_attend", q, n, 0, dim, on)
    heads = q.shape[1]
    if out is None:
        out = _empty(q.shape, torch.bfloat16, q.device, stream)
    ro = _rows("ecfa_attend", out, n, heads, dim, on)
    opts = _opts("ecfa_attend", cache, batch, heads, scale, causal, window, softcap, slopes, prefix)
    if workspace is None:
        workspace = attend_workspace(cache, batch, heads, stream)
    elif workspace.get_device() != on or not workspace.is_contiguous():
        raise _bad("ecfa_attend")
    rc = _attend(cache.c, batch.c, opts, rq, ro, None if workspace is None else workspace.data_ptr(),
                 0 if workspace is None else workspace.numel(), at)
    if rc:
        _e._check("ecfa_attend", rc)
    return out


def ecfa_quant(x, group=0, q=None, scale=None, stream=None):
    """x (rows, cols) fp32 or BF16, rows of any stride, to (E4M3 (rows, cols), fp32 scales (rows,) or with group = 128 (rows, cols / 128));
    the result is a ``torch.float8_e4m3fn`` tensor unless q is given (uint8 or float8_e4m3fn, dense)."""
    shape, dtype = x.shape, _DTYPE.get(x.dtype)
    if len(shape) != 2 or dtype is None or group not in (0, 128):
        raise _bad("ecfa_quant")
    rows, cols = shape
    on = x.get_device()
    at = _stream_ptr("ecfa_quant", on, stream)
    row_stride, one = x.stride()
    if cols > 1 and one != 1:
        raise _bad("ecfa_quant")
    want = (rows, cols // 128) if group else (rows,)
    if q is None:
        q = _empty((rows, cols), torch.float8_e4m3fn, x.device, stream)
    if scale is None:
        scale = _empty(want, torch.float32, x.device, stream)
    if (q.dtype not in _BYTES or q.shape != shape or not q.is_contiguous() or scale.dtype != torch.float32 or scale.shape != want
            or not scale.is_contiguous() or q.get_device() != on or scale.get_device() != on):
        raise _bad("ecfa_quant")
    rc = _quant(x.data_ptr(), dtype, rows, cols, row_stride, group, q.data_ptr(), scale.data_ptr(), at)
    if rc:
        _e._check("ecfa_quant", rc)
    return q, scale
