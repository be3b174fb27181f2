"""Rotary positions, a paged key/value cache and attention over it, on AMD Instinct MI355X.

The same kind of binding as ``seq.py`` over the same library (``include/im2win_seq.h``): no fallback, nothing recorded by
autograd, ``stream`` as there.  Tensors on another device than the current one make the call run on that device.

    freq = seq_rotary_frequencies(rot, base=10000.0, factor=8.0, trained=4096)    # host fp64 [rot/2], kept by the caller
    y = seq_rotary_forward(x, freq, positions)                                    # x [B][L][H][D]
    dx = seq_rotary_backward(dy, freq, positions)
    seq_cache_write(k, v, k_pages, v_pages, table, start, count)                  # pages [pages][page][Hkv][D]
    k, v = seq_cache_read(k_pages, v_pages, table, length, L)                     # [B][L][Hkv][D]
    out, lse = seq_paged_attention_forward(q, k_pages, v_pages, table, length)    # q [B][H][D]

Pages hold the type of the keys, or ``torch.int8`` / ``torch.float8_e4m3fn`` codes beside fp32 scales
[pages][page][Hkv] (``k_scale``, ``v_scale``).
"""
from __future__ import annotations

import ctypes
import struct

from . import _check, _i64, _nbytes, _vp, Im2winError
from .seq import _elsewhere, _library as _seq_library, _like, _same_device

__all__ = ["seq_rotary_frequencies", "seq_rotary_forward", "seq_rotary_backward", "seq_cache_write", "seq_cache_read",
           "seq_paged_attention_workspace_bytes", "seq_paged_attention_forward"]

_int = ctypes.c_int
# seq_rotary_t: dt, interleaved, by_token, amplitude; B, L, H, D, rot; strides of x, y; positions, freq
_ROTARY = struct.Struct("@3if11q2P")
# seq_cache_t: dt; B, pages, page, max_pages, Hkv, D; strides of k, v, their scales; table's; k, v, scales, table
_CACHE = struct.Struct("@i4x19q5P")
# seq_paged_attention_t: dt, scale, cap; H; strides of q, out; R, strip, len
_PAGED = struct.Struct("@i2f4x6q2P")
_TRIPLE = struct.Struct("@3q")

# Most of a small call is this file's: attributes of tensors are read once and
# compared inline, and what torch looks up by name is kept here from the first
# call on (torch is not imported with the package).
_lib = _torch = _codes = _int32 = _float32 = _float64 = _device = _raw_stream = None


def _library():
    if _lib is None:
        _load()
    return _lib


def _load():
    global _lib, _torch, _codes, _int32, _float32, _float64
    import torch
    lib = _seq_library()
    text = ctypes.c_char_p
    lib.seq_rotary_forward.restype = lib.seq_rotary_backward.restype = _int
    lib.seq_rotary_forward.argtypes = lib.seq_rotary_backward.argtypes = [text, _vp, _vp, _vp]
    lib.seq_rotary_frequencies.restype = _int
    lib.seq_rotary_frequencies.argtypes = [_vp, _i64] + [ctypes.c_double] * 5
    lib.seq_cache_write.restype = lib.seq_cache_read.restype = _int
    lib.seq_cache_write.argtypes = [text, _vp, _vp, text, text, _i64, _int, _vp, _vp, _vp]
    lib.seq_cache_read.argtypes = [text, _vp, _vp, text, text, _i64, _int, _vp, _vp]
    lib.seq_paged_attention_workspace_bytes.restype = _i64
    lib.seq_paged_attention_workspace_bytes.argtypes = [text, _i64, _int]
    lib.seq_paged_attention_forward.restype = _int
    lib.seq_paged_attention_forward.argtypes = [text, text, _vp, _vp, _vp, _vp, _i64, _vp]
    _torch, _int32, _float32, _float64 = torch, torch.int32, torch.float32, torch.float64
    # cache elements of 8 bits have codes from 16 on
    _codes = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.int8: 16, torch.float8_e4m3fn: 17}
    _lib = lib


def _place(t):
    """(whether ``t`` lies on another GPU than the current one, the handle of
    the current stream): as torch.cuda.current_device and current_stream say,
    without building their objects (3 us)."""
    global _device, _raw_stream
    at = t.get_device()
    if at < 0:  # no GPU's memory: the library refuses it
        return False, 0
    if _device is None:
        _torch.cuda.current_device()  # initialises
        _device, _raw_stream = _torch._C._cuda_getDevice, _torch._C._cuda_getCurrentRawStream
    if at != _device():
        return True, 0
    return False, _raw_stream(at)


def _over_there(t, call, *args):
    with _torch.cuda.device(t.device):
        return call(*args)


def _code(dtype) -> int:
    code = _codes.get(dtype)
    if code is None:
        raise ValueError("no operator here takes elements of type %s" % dtype)
    return code


def seq_rotary_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, trained: float = 0.0, low: float = 1.0,
                           high: float = 32.0):
    """Frequencies [rot/2] (host, fp64) of pairs of channels: base ** (-2i/rot),
    for contexts ``factor`` times as long as the ``trained`` one slowed down by
    ``factor`` where a pair turns at most ``low`` times within it, kept where it
    turns at least ``high`` times, on a straight line between; trained 0: all
    slowed down."""
    _library()
    freq = _torch.empty(rot // 2 if rot > 1 else 1, dtype=_float64)
    _check(_lib.seq_rotary_frequencies(freq.data_ptr(), rot, base, factor, trained, low, high), "seq_rotary_frequencies")
    return freq


def _rotary(call, what, x, freq, positions, interleaved, amplitude, out, stream):
    xs, st, device = x.shape, x.stride(), x.device
    if len(xs) != 4:
        raise ValueError("x must have four dimensions")
    B, L, H, D = xs
    if st[3] != 1 and D > 1:
        raise ValueError("x must be dense in its last dimension")
    if freq.dim() != 1 or freq.dtype != _float64 or freq.is_cuda or not freq.is_contiguous():
        raise ValueError("freq must be a contiguous fp64 [rot/2] tensor in host memory")
    if out is None:
        out = _torch.empty_like(x)
    else:
        _like(out, xs, x.dtype, "out")
        _same_device(x, out)
    so = out.stride()
    if so[3] != 1 and D > 1:
        raise ValueError("out must be dense in its last dimension")
    pos = by_token = 0
    if positions is not None:
        by_token = 1 if positions.dim() == 2 else 0
        if positions.shape != ((B, L) if by_token else (B,)) or positions.dtype != _int32 or not positions.is_contiguous():
            raise ValueError("positions must be a contiguous int32 [B] or [B][L] tensor")
        if positions.device != device:
            raise ValueError("all tensors must be on %s" % device)
        pos = positions.data_ptr()
    a = _ROTARY.pack(_code(x.dtype), 1 if interleaved else 0, by_token, amplitude, B, L, H, D, 2 * freq.shape[0], st[0],
                     st[1], st[2], so[0], so[1], so[2], pos, freq.data_ptr())
    rc = call(a, x.data_ptr(), out.data_ptr(), stream)
    if rc:
        raise Im2winError(rc, what)
    return out


def seq_rotary_forward(x, freq, positions=None, interleaved: bool = False, amplitude: float = 1.0, out=None, stream=None):
    """Turns the pairs of the first ``2 * len(freq)`` channels of each head of
    ``x`` [B][L][H][D] (any strides, the last dimension dense) by the angles
    position * freq; the other channels are copied.

    positions    int32 [B][L], or [B] of each sequence's first token; None: 0, 1, ..
    interleaved  pairs are channels (2i, 2i+1), else (i, i + rot/2)
    amplitude    factor of the turned channels
    out          like ``x``, any strides; may be ``x``
    """
    if stream is not None:
        return _elsewhere(stream, seq_rotary_forward, x, freq, positions, interleaved, amplitude, out)
    call = _library().seq_rotary_forward
    away, handle = _place(x)
    if away:
        return _over_there(x, seq_rotary_forward, x, freq, positions, interleaved, amplitude, out)
    return _rotary(call, "seq_rotary_forward", x, freq, positions, interleaved, amplitude, out, handle)


def seq_rotary_backward(dy, freq, positions=None, interleaved: bool = False, amplitude: float = 1.0, out=None, stream=None):
    """The gradient of ``seq_rotary_forward``'s input from that of its result."""
    if stream is not None:
        return _elsewhere(stream, seq_rotary_backward, dy, freq, positions, interleaved, amplitude, out)
    call = _library().seq_rotary_backward
    away, handle = _place(dy)
    if away:
        return _over_there(dy, seq_rotary_backward, dy, freq, positions, interleaved, amplitude, out)
    return _rotary(call, "seq_rotary_backward", dy, freq, positions, interleaved, amplitude, out, handle)


def _cache(k, v, table, k_scale, v_scale):
    """The packed description of a cache, its element code, device, B and the
    pages' shape."""
    ks, sk, sv, ts, st = k.shape, k.stride(), v.stride(), table.shape, table.stride()
    dtype, device = k.dtype, k.device
    if len(ks) != 4 or v.shape != ks or v.dtype != dtype:
        raise ValueError("k_pages and v_pages must have one shape [pages][page][Hkv][D] and one type")
    pages, page, Hkv, D = ks
    if (sk[3] != 1 or sv[3] != 1) and D > 1:
        raise ValueError("k_pages and v_pages must be dense in their last dimension")
    if len(ts) != 2 or table.dtype != _int32 or (st[1] != 1 and ts[1] > 1):
        raise ValueError("table must be an int32 [B][max_pages] tensor, dense in its last dimension")
    B, most = ts
    if v.device != device or table.device != device:
        raise ValueError("all tensors must be on %s" % device)
    code = _code(dtype)
    if code < 16:
        if k_scale is not None or v_scale is not None:
            raise ValueError("k_scale and v_scale go with 8-bit pages")
        return _CACHE.pack(code, B, pages, page, most, Hkv, D, sk[0], sk[1], sk[2], sv[0], sv[1], sv[2], 0, 0, 0, 0, 0, 0,
                           st[0] if B > 1 else most, k.data_ptr(), v.data_ptr(), 0, 0, table.data_ptr()), code, device, B, ks
    if k_scale is None or v_scale is None:
        raise ValueError("8-bit pages need k_scale and v_scale")
    shape = ks[:3]
    if k_scale.shape != shape or v_scale.shape != shape or k_scale.dtype != _float32 or v_scale.dtype != _float32:
        raise ValueError("k_scale and v_scale must be fp32 [pages][page][Hkv]")
    if k_scale.device != device or v_scale.device != device:
        raise ValueError("all tensors must be on %s" % device)
    return _CACHE.pack(code, B, pages, page, most, Hkv, D, sk[0], sk[1], sk[2], sv[0], sv[1], sv[2], *k_scale.stride(),
                       *v_scale.stride(), st[0] if B > 1 else most, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                       v_scale.data_ptr(), table.data_ptr()), code, device, B, ks


def _counts(name, t, B, device):
    if t.dtype != _int32 or t.dim() != 1 or t.shape[0] != B or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 [%d] tensor" % (name, B))
    if t.device != device:
        raise ValueError("all tensors must be on %s" % device)
    return t.data_ptr()


def _dense(k, v, L, device, B, ps):
    """Strides of k and v [B][L][Hkv][D], packed."""
    shape, sk, sv = k.shape, k.stride(), v.stride()
    if len(shape) != 4 or shape[0] != B or shape[1] != L or shape[2] != ps[2] or shape[3] != ps[3] or v.shape != shape:
        raise ValueError("k and v must be [B][L][Hkv][D], as the table and the pages have it")
    if v.dtype != k.dtype:
        raise TypeError("k and v must have one type")
    if (sk[3] != 1 or sv[3] != 1) and ps[3] > 1:
        raise ValueError("k and v must be dense in their last dimension")
    if k.device != device or v.device != device:
        raise ValueError("all tensors must be on %s" % device)
    return _TRIPLE.pack(sk[0], sk[1], sk[2]), _TRIPLE.pack(sv[0], sv[1], sv[2])


def seq_cache_write(k, v, k_pages, v_pages, table, start=None, count=None, k_scale=None, v_scale=None, stream=None):
    """Writes the tokens k, v [B][L][Hkv][D] (any strides, the last dimension
    dense) into the pages: token t < count[b] of sequence b becomes its token
    start[b] + t.

    k_pages, v_pages  [pages][page][Hkv][D], any strides with a dense last dimension
    table    int32 [B][max_pages]: each sequence's pages in order; entries that name no page take nothing
    start    int32 [B], None: 0;  count  int32 [B], None: all L
    k_scale, v_scale  fp32 [pages][page][Hkv], written with 8-bit pages
    """
    if stream is not None:
        return _elsewhere(stream, seq_cache_write, k, v, k_pages, v_pages, table, start, count, k_scale, v_scale)
    call = _library().seq_cache_write
    away, handle = _place(k)
    if away:
        return _over_there(k, seq_cache_write, k, v, k_pages, v_pages, table, start, count, k_scale, v_scale)
    c, code, device, B, ps = _cache(k_pages, v_pages, table, k_scale, v_scale)
    L = k.shape[1] if k.dim() == 4 else -1
    sk, sv = _dense(k, v, L, device, B, ps)
    dt = _code(k.dtype)
    if dt >= 16 or (code < 16 and dt != code):
        raise TypeError("k and v must have the type of the pages, or a wider one than 8-bit pages")
    first = 0 if start is None else _counts("start", start, B, device)
    n = 0 if count is None else _counts("count", count, B, device)
    rc = call(c, k.data_ptr(), v.data_ptr(), sk, sv, L, dt, first, n, handle)
    if rc:
        raise Im2winError(rc, "seq_cache_write")


def seq_cache_read(k_pages, v_pages, table, length, L: int, dtype=None, k_scale=None, v_scale=None, k=None, v=None,
                   stream=None):
    """The first length[b] tokens of each sequence as dense (k, v), each
    [B][L][Hkv][D] of type ``dtype`` (that of the pages; fp32 for 8-bit ones),
    written to ``k`` and ``v`` where given; rows from length[b] on are zeros."""
    if stream is not None:
        return _elsewhere(stream, seq_cache_read, k_pages, v_pages, table, length, L, dtype, k_scale, v_scale, k, v)
    call = _library().seq_cache_read
    away, handle = _place(k_pages)
    if away:
        return _over_there(k_pages, seq_cache_read, k_pages, v_pages, table, length, L, dtype, k_scale, v_scale, k, v)
    c, code, device, B, ps = _cache(k_pages, v_pages, table, k_scale, v_scale)
    if dtype is None:
        dtype = k_pages.dtype if code < 16 else _float32
    dt = _code(dtype)
    if dt >= 16 or (code < 16 and dt != code):
        raise TypeError("dtype must be that of the pages, or a wider one than 8-bit pages")
    if k is None:
        k = _torch.empty((B, L, ps[2], ps[3]), dtype=dtype, device=device)
    elif k.dtype != dtype:
        raise ValueError("k and v must have the type %s" % dtype)
    if v is None:
        v = _torch.empty_like(k, memory_format=_torch.contiguous_format)
    sk, sv = _dense(k, v, L, device, B, ps)
    n = _counts("length", length, B, device)
    rc = call(c, k.data_ptr(), v.data_ptr(), sk, sv, L, dt, n, handle)
    if rc:
        raise Im2winError(rc, "seq_cache_read")
    return k, v


def _paged_ws(c, H, dt):
    n = _lib.seq_paged_attention_workspace_bytes(c, H, dt)
    if n < 0:
        raise Im2winError(int(n), "seq_paged_attention_workspace_bytes")
    return n


def seq_paged_attention_workspace_bytes(q, k_pages, v_pages, table, k_scale=None, v_scale=None) -> int:
    """Bytes of workspace of ``seq_paged_attention_forward`` with these operands."""
    _library()
    return _paged_ws(_cache(k_pages, v_pages, table, k_scale, v_scale)[0], q.shape[1], _code(q.dtype))


def seq_paged_attention_forward(q, k_pages, v_pages, table, length, scale=None, cap: float = 0.0, bias=None, k_scale=None,
                                v_scale=None, out=None, ws=None, stream=None):
    """Attention of one new token of each sequence, q [B][H][D] (any strides,
    the last dimension dense), the last of its length[b] tokens, over the pages.
    Returns (out like q, lse [B][H] fp32); scale, cap and bias as in
    ``seq_attention_forward``, pages and table as in ``seq_cache_write``."""
    if stream is not None:
        return _elsewhere(stream, seq_paged_attention_forward, q, k_pages, v_pages, table, length, scale, cap, bias,
                          k_scale, v_scale, out, ws)
    call = _library().seq_paged_attention_forward
    away, handle = _place(q)
    if away:
        return _over_there(q, seq_paged_attention_forward, q, k_pages, v_pages, table, length, scale, cap, bias, k_scale,
                           v_scale, out, ws)
    c, code, device, B, ps = _cache(k_pages, v_pages, table, k_scale, v_scale)
    qs, sq, dt = q.shape, q.stride(), _code(q.dtype)
    if len(qs) != 3 or qs[0] != B or qs[2] != ps[3]:
        raise ValueError("q must be [B][H][D], as the table and the pages have it")
    if dt >= 16 or (code < 16 and dt != code):
        raise TypeError("q must have the type of the pages, or a wider one than 8-bit pages")
    H, D = qs[1], qs[2]
    if sq[2] != 1 and D > 1:
        raise ValueError("q must be dense in its last dimension")
    if q.device != device:
        raise ValueError("all tensors must be on %s" % device)
    if out is None:
        out = _torch.empty_like(q)
    else:
        _like(out, qs, q.dtype, "out")
        _same_device(q, out)
    so = out.stride()
    if so[2] != 1 and D > 1:
        raise ValueError("out must be dense in its last dimension")
    n = _counts("length", length, B, device)
    R = strip = 0
    if bias is not None:
        if bias.dim() != 2 or bias.shape[0] != H or bias.shape[1] % 2 == 0 or bias.shape[1] < 3 \
                or bias.dtype != _float32 or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous fp32 [H][2R+1] strip")
        _same_device(q, bias)
        R, strip = bias.shape[1] // 2, bias.data_ptr()
    a = _PAGED.pack(dt, D ** -0.5 if scale is None else scale, cap, H, sq[0], sq[1], so[0], so[1], R, strip, n)
    lse = _torch.empty((B, H), dtype=_float32, device=device)
    if ws is not None:
        _same_device(q, ws)
        at, size = ws.data_ptr(), _nbytes(ws)
    else:
        at, size = 0, _paged_ws(c, H, dt)
        if size:
            ws = _torch.empty(size, dtype=_torch.uint8, device=device)
            at = ws.data_ptr()
    rc = call(c, a, q.data_ptr(), out.data_ptr(), lse.data_ptr(), at, size, handle)
    if rc:
        raise Im2winError(rc, "seq_paged_attention_forward")
    return out, lse
