"""Sequence operators on AMD Instinct MI355X: layer norm, relative position bias, attention.

A thin binding over the calls of ``include/im2win_seq.h`` in ``libim2win.so``: shapes, strides and device pointers of
PyTorch tensors and the current HIP stream.  Outputs and workspaces that are not given are allocated; there is no
fallback.  With ``stream`` (a torch stream or a handle) the call is made as under ``torch.cuda.stream(stream)``: its
inputs have to be ready there, and its results are first ready there.  As with the convolutions, autograd does not
record the calls: results are detached also where inputs require gradients, which the backward calls compute
(``examples/conv_tokens.py`` wraps them in ``torch.autograd.Function``).

    y, mean, rstd = seq_layer_norm_forward(x, weight, bias, eps)
    dx, dweight, dbias = seq_layer_norm_backward(dy, x, weight, mean, rstd)
    strip = seq_rel_bias_forward(table, max_distance, two_sided=True)         # [H][2R+1] by distance
    dtable = seq_rel_bias_backward(dstrip, buckets, two_sided=True)           # dstrip [H][2R+1] or [n][H][2R+1]
    out, lse = seq_attention_forward(q, k, v, bias=strip, causal=True)        # q [B][Lq][H][D], k, v [B][Lk][Hkv][D]
    dq, dk, dv, dstrip = seq_attention_backward(dout, q, k, v, out, lse, bias=strip, causal=True)
"""
from __future__ import annotations

import ctypes
import struct

from . import _check, _dtype_code, _i64, _nbytes, _stream, _vp, load_library, Im2winError

__all__ = ["seq_layer_norm_workspace_bytes", "seq_layer_norm_forward", "seq_layer_norm_backward", "seq_rel_bias_bucket",
           "seq_rel_bias_forward", "seq_rel_bias_backward", "seq_attention_workspace_bytes", "seq_attention_forward",
           "seq_attention_backward"]

_lib = None
_int = ctypes.c_int


# seq_attention_t: dt, causal, align_end, scale, cap; B, Lq, Lk, H, Hkv, D; eight operands' strides (q, k, v, out, dout,
# dq, dk, dv); R, strip, kv_len, prefix, q_doc, k_doc.  One pack takes 1 us, a ctypes structure set field by field 6.
_PACK = struct.Struct("@3i2f4x6q24qq5P")
_NO_STRIDES = (0, 0, 0)


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        lib.seq_layer_norm_forward.restype = _int
        lib.seq_layer_norm_forward.argtypes = [_vp] * 6 + [_i64] * 3 + [ctypes.c_float, _int, _int, _vp]
        lib.seq_layer_norm_workspace_bytes.restype = _i64
        lib.seq_layer_norm_workspace_bytes.argtypes = [_i64] * 2
        lib.seq_layer_norm_backward.restype = _int
        lib.seq_layer_norm_backward.argtypes = [_vp] * 9 + [_i64] * 5 + [_int, _int, _vp]
        lib.seq_rel_bias_forward.restype = _int
        lib.seq_rel_bias_forward.argtypes = [_vp] * 2 + [_i64] * 3 + [_int, _int, _vp]
        lib.seq_rel_bias_backward.restype = _int
        lib.seq_rel_bias_backward.argtypes = [_vp] * 2 + [_i64] * 4 + [_int, _int, _vp]
        lib.seq_rel_bias_bucket.restype = _i64
        lib.seq_rel_bias_bucket.argtypes = [_i64] * 3 + [_int]
        lib.seq_attention_workspace_bytes.restype = _i64
        lib.seq_attention_workspace_bytes.argtypes = [ctypes.c_char_p, _int]
        lib.seq_attention_forward.restype = _int
        lib.seq_attention_forward.argtypes = [ctypes.c_char_p] + [_vp] * 6 + [_i64, _vp]
        lib.seq_attention_backward.restype = _int
        lib.seq_attention_backward.argtypes = [ctypes.c_char_p] + [_vp] * 11 + [_i64, _vp]
        _lib = lib
    return _lib


def _elsewhere(stream, call, *args):
    """``call`` with ``stream`` as the current stream, so that what it allocates
    comes from that stream's memory: a block that was freed on the caller's
    stream may still be in use by work pending there.  The caller's tensors are
    recorded on the call's stream and its results on the caller's, so that
    neither is reused before the other stream's work on it has ended."""
    import torch
    s = torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream
    here = torch.cuda.current_stream(s.device)
    with torch.cuda.stream(s):
        res = call(*args)
    for t in args:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(s)
    for t in res if isinstance(res, tuple) else (res,):
        if t is not None:
            t.record_stream(here)
    return res


def _rows(x, what):
    """(rows, C, stride) of a tensor whose last dimension is dense and whose
    other dimensions step evenly."""
    if x.dim() == 0:
        raise ValueError("%s must have a channel dimension" % what)
    C = x.shape[-1]
    try:
        flat = x if x.dim() == 2 else x.view(-1, C)
    except RuntimeError:
        raise ValueError("%s must have evenly spaced rows (one stride over its leading dimensions)" % what) from None
    if C > 1 and flat.stride(1) != 1:
        raise ValueError("%s must be dense in its last dimension" % what)
    return flat.shape[0], C, flat.stride(0) if flat.shape[0] > 1 else C


def _params(C, dtype, *params):
    import torch
    wdt = params[0].dtype
    for p in params:
        if p.dim() != 1 or p.shape[0] != C or not p.is_contiguous():
            raise ValueError("weight and bias must be contiguous [%d] tensors" % C)
        if p.dtype != wdt or wdt not in (dtype, torch.float32):
            raise TypeError("weight and bias must both have the rows' type or fp32")
    return _dtype_code(wdt)


def _same_device(first, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("all tensors must be on %s" % first.device)


def seq_layer_norm_workspace_bytes(rows: int, C: int) -> int:
    n = _library().seq_layer_norm_workspace_bytes(rows, C)
    if n < 0:
        raise Im2winError(int(n), "seq_layer_norm_workspace_bytes")
    return int(n)


def seq_layer_norm_forward(x, weight, bias, eps: float = 1e-5, out=None, stream=None):
    """Layer norm over the last dimension.  Returns (y, mean, rstd): y dense
    like ``x`` (written to ``out`` when given, which may be a dense ``x``),
    the statistics fp32 with a value per row."""
    if stream is not None:
        return _elsewhere(stream, seq_layer_norm_forward, x, weight, bias, eps, out)
    import torch
    rows, C, xs = _rows(x, "x")
    wdt = _params(C, x.dtype, weight, bias)
    _same_device(x, weight, bias, out)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    if y.shape != x.shape or y.dtype != x.dtype or not y.is_contiguous():
        raise ValueError("out must be contiguous, with the shape and type of x")
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    _check(_library().seq_layer_norm_forward(x.data_ptr(), weight.data_ptr(), bias.data_ptr(), y.data_ptr(),
                                             mean.data_ptr(), rstd.data_ptr(), rows, C, xs, eps, _dtype_code(x.dtype),
                                             wdt, _stream(None)), "seq_layer_norm_forward")
    return y, mean, rstd


def seq_layer_norm_backward(dy, x, weight, mean, rstd, ws=None, stream=None):
    """Gradients of the layer norm: (dx, dweight, dbias)."""
    if stream is not None:
        return _elsewhere(stream, seq_layer_norm_backward, dy, x, weight, mean, rstd, ws)
    import torch
    rows, C, xs = _rows(x, "x")
    rows2, C2, dys = _rows(dy, "dy")
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have the shape and type of x")
    wdt = _params(C, x.dtype, weight)
    for t in (mean, rstd):
        if t.numel() != rows or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("mean and rstd must be contiguous fp32, a value per row")
    _same_device(x, dy, weight, mean, rstd, ws)
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw, db = torch.empty_like(weight), torch.empty_like(weight)
    if ws is None:
        ws = torch.empty(seq_layer_norm_workspace_bytes(rows, C), dtype=torch.uint8, device=x.device)
    _check(_library().seq_layer_norm_backward(dy.data_ptr(), x.data_ptr(), weight.data_ptr(), mean.data_ptr(),
                                              rstd.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(),
                                              ws.data_ptr(), _nbytes(ws), rows, C, dys, xs, _dtype_code(x.dtype), wdt,
                                              _stream(None)), "seq_layer_norm_backward")
    return dx, dw, db


def seq_rel_bias_bucket(distance: int, buckets: int, max_distance: int, two_sided: bool = True) -> int:
    """The bucket of a distance (key position minus query position)."""
    b = _library().seq_rel_bias_bucket(distance, buckets, max_distance, 1 if two_sided else 0)
    if b < 0:
        raise Im2winError(int(b), "seq_rel_bias_bucket")
    return int(b)


def seq_rel_bias_forward(table, max_distance: int, two_sided: bool = True, out=None, stream=None):
    """The strip [H][2*max_distance + 1] (fp32) of a bucket table [buckets][H]."""
    if stream is not None:
        return _elsewhere(stream, seq_rel_bias_forward, table, max_distance, two_sided, out)
    import torch
    if table.dim() != 2 or not table.is_contiguous():
        raise ValueError("table must be a contiguous [buckets][H] tensor")
    buckets, H = table.shape
    shape = (H, 2 * max_distance + 1)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=table.device)
    if tuple(out.shape) != shape or out.dtype != torch.float32 or not out.is_contiguous():
        raise ValueError("out must be a contiguous fp32 [H][2*max_distance + 1] tensor")
    _same_device(table, out)
    _check(_library().seq_rel_bias_forward(table.data_ptr(), out.data_ptr(), H, buckets, max_distance,
                                           1 if two_sided else 0, _dtype_code(table.dtype), _stream(None)),
           "seq_rel_bias_forward")
    return out


def seq_rel_bias_backward(dstrip, buckets: int, two_sided: bool = True, dtype=None, stream=None):
    """The table's gradient [buckets][H] (of type ``dtype``, fp32 by default)
    from strips' gradients [H][2R+1], or [n][H][2R+1] of n layers that share
    the table."""
    if stream is not None:
        return _elsewhere(stream, seq_rel_bias_backward, dstrip, buckets, two_sided, dtype)
    import torch
    if dstrip.dim() not in (2, 3) or dstrip.dtype != torch.float32 or not dstrip.is_contiguous():
        raise ValueError("dstrip must be a contiguous fp32 [H][2R+1] or [n][H][2R+1] tensor")
    n = dstrip.shape[0] if dstrip.dim() == 3 else 1
    H, width = dstrip.shape[-2:]
    if width % 2 == 0:
        raise ValueError("dstrip must hold an odd number of distances, -R .. R")
    dtype = torch.float32 if dtype is None else dtype
    dtable = torch.empty((buckets, H), dtype=dtype, device=dstrip.device)
    _check(_library().seq_rel_bias_backward(dstrip.data_ptr(), dtable.data_ptr(), n, H, buckets, width // 2,
                                            1 if two_sided else 0, _dtype_code(dtype), _stream(None)),
           "seq_rel_bias_backward")
    return dtable


def _strides(t, what):
    """Strides of the sequence, token and head dimensions."""
    st = t.stride()
    if len(st) != 4:
        raise ValueError("%s must have four dimensions" % what)
    if st[3] != 1 and t.shape[3] > 1:
        raise ValueError("%s must be dense in its last dimension" % what)
    return st[:3]


def _dense(shape):
    return (shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])


def _ints(name, t, shape, device):
    import torch
    if t.shape != shape or t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s" % (name, shape))
    if t.device != device:
        raise ValueError("all tensors must be on %s" % device)
    return t.data_ptr()


def _describe(q, k, v, strides, scale, cap, causal, align_end, bias, kv_len, prefix, q_doc, k_doc):
    """The packed description of a call; ``strides``: of out, dout, dq, dk, dv."""
    qs, ks = q.shape, k.shape
    if len(qs) != 4 or len(ks) != 4:
        raise ValueError("q must be [B][Lq][H][D], k and v [B][Lk][Hkv][D]")
    B, Lq, H, D = qs
    _, Lk, Hkv, _ = ks
    if v.shape != ks or ks[0] != B or ks[3] != D:
        raise ValueError("k and v must have one shape, with the batch and channels of q")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k and v must have one type")
    device = q.device
    if k.device != device or v.device != device:
        raise ValueError("all tensors must be on %s" % device)
    R = strip = lens = pre = qd = kd = 0
    if bias is not None:
        import torch
        if bias.dim() != 2 or bias.shape[0] != H or bias.shape[1] % 2 == 0 or bias.shape[1] < 3 \
                or bias.dtype != torch.float32 or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous fp32 [H][2R+1] strip")
        if bias.device != device:
            raise ValueError("all tensors must be on %s" % device)
        R, strip = bias.shape[1] // 2, bias.data_ptr()
    if kv_len is not None:
        lens = _ints("kv_len", kv_len, (B,), device)
    if prefix is not None:
        if not causal:
            raise ValueError("prefix needs causal")
        pre = _ints("prefix", prefix, (B,), device)
    if q_doc is not None or k_doc is not None:
        if q_doc is None or k_doc is None:
            raise ValueError("q_doc and k_doc go together")
        qd, kd = _ints("q_doc", q_doc, (B, Lq), device), _ints("k_doc", k_doc, (B, Lk), device)
    so, sdo, sdq, sdk, sdv = strides
    return _PACK.pack(_dtype_code(q.dtype), 1 if causal else 0, 1 if align_end else 0, D ** -0.5 if scale is None else scale,
                      cap, B, Lq, Lk, H, Hkv, D, *_strides(q, "q"), *_strides(k, "k"), *_strides(v, "v"), *so, *sdo, *sdq,
                      *sdk, *sdv, R, strip, lens, pre, qd, kd)


def _attention_ws(a, backward, ws, device):
    n = _library().seq_attention_workspace_bytes(a, backward)
    if n < 0:
        raise Im2winError(int(n), "seq_attention_workspace_bytes")
    if ws is None and n:
        import torch
        ws = torch.empty(int(n), dtype=torch.uint8, device=device)
    return ws


def seq_attention_workspace_bytes(q, k, v, backward: bool = False, **options) -> int:
    """Bytes of workspace of the forward or backward call with these operands
    and the options of ``seq_attention_forward``."""
    opts = dict(scale=None, cap=0.0, causal=False, align_end=False, bias=None, kv_len=None, prefix=None, q_doc=None,
                k_doc=None)
    opts.update(options)
    like_q, like_k = _dense(q.shape), _dense(k.shape)
    a = _describe(q, k, v, (like_q, like_q, like_q, like_k, like_k), **opts)
    n = _library().seq_attention_workspace_bytes(a, 1 if backward else 0)
    if n < 0:
        raise Im2winError(int(n), "seq_attention_workspace_bytes")
    return int(n)


def _like(t, shape, dtype, what):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s must have shape %s and type %s" % (what, tuple(shape), dtype))


def seq_attention_forward(q, k, v, scale=None, cap: float = 0.0, causal: bool = False, align_end: bool = False, bias=None,
                          kv_len=None, prefix=None, q_doc=None, k_doc=None, out=None, ws=None, stream=None):
    """Attention of q [B][Lq][H][D] over k, v [B][Lk][Hkv][D] (any strides, the
    last dimension dense).  Returns (out like q, lse [B][H][Lq] fp32).

    scale     of the products, D ** -0.5 by default;  cap: scores become cap*tanh(score/cap), 0: as they are
    causal    a query sees no later key, except the first prefix[b] keys
    align_end queries are the last Lq of a sequence's positions (else the first)
    bias      strip [H][2R+1] added by clamped distance (seq_rel_bias_forward)
    kv_len    [B] int32: keys from there on do not exist
    q_doc, k_doc  [B][Lq], [B][Lk] int32: pairs need equal ids, negative ids see and are seen by nothing
    """
    if stream is not None:
        return _elsewhere(stream, seq_attention_forward, q, k, v, scale, cap, causal, align_end, bias, kv_len, prefix,
                          q_doc, k_doc, out, ws)
    import torch
    device = q.device
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=device)
    else:
        _like(out, q.shape, q.dtype, "out")
        _same_device(q, out)
    a = _describe(q, k, v, (_strides(out, "out"), _NO_STRIDES, _NO_STRIDES, _NO_STRIDES, _NO_STRIDES), scale, cap, causal,
                  align_end, bias, kv_len, prefix, q_doc, k_doc)
    lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=device)
    ws = _attention_ws(a, 0, ws, device)
    _check(_library().seq_attention_forward(a, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                            *_workspace(q, ws), _stream(None)), "seq_attention_forward")
    return out, lse


def _workspace(like, ws):
    if ws is None:
        return None, 0
    _same_device(like, ws)
    return ws.data_ptr(), _nbytes(ws)


def seq_attention_backward(dout, q, k, v, out, lse, scale=None, cap: float = 0.0, causal: bool = False,
                           align_end: bool = False, bias=None, kv_len=None, prefix=None, q_doc=None, k_doc=None, dq=None,
                           dk=None, dv=None, ws=None, stream=None):
    """Gradients (dq, dk, dv, dstrip) of ``seq_attention_forward`` with the same
    options, from its ``out`` and ``lse``; dstrip is None without a bias.  dq,
    dk and dv are written to the tensors given, of any strides with a dense
    last dimension (columns of one packed tensor, for example)."""
    if stream is not None:
        return _elsewhere(stream, seq_attention_backward, dout, q, k, v, out, lse, scale, cap, causal, align_end, bias,
                          kv_len, prefix, q_doc, k_doc, dq, dk, dv, ws)
    import torch
    _like(dout, q.shape, q.dtype, "dout")
    _like(out, q.shape, q.dtype, "out")
    _like(lse, (q.shape[0], q.shape[2], q.shape[1]), torch.float32, "lse")
    if not lse.is_contiguous():
        raise ValueError("lse must be contiguous")
    device = q.device
    dq = torch.empty(q.shape, dtype=q.dtype, device=device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=q.dtype, device=device) if dk is None else dk
    dv = torch.empty(v.shape, dtype=q.dtype, device=device) if dv is None else dv
    _like(dq, q.shape, q.dtype, "dq")
    _like(dk, k.shape, q.dtype, "dk")
    _like(dv, v.shape, q.dtype, "dv")
    _same_device(q, dout, out, lse, dq, dk, dv)
    a = _describe(q, k, v, (_strides(out, "out"), _strides(dout, "dout"), _strides(dq, "dq"), _strides(dk, "dk"),
                            _strides(dv, "dv")), scale, cap, causal, align_end, bias, kv_len, prefix, q_doc, k_doc)
    dstrip = None if bias is None else torch.empty(bias.shape, dtype=torch.float32, device=device)
    ws = _attention_ws(a, 1, ws, device)
    _check(_library().seq_attention_backward(a, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                             lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                             None if dstrip is None else dstrip.data_ptr(), *_workspace(q, ws),
                                             _stream(None)), "seq_attention_backward")
    return dq, dk, dv, dstrip
