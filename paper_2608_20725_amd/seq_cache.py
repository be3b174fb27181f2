"""Rotary positions, a paged key/value cache and attention over it, on AMD Instinct MI355X.

The calls of ``include/im2win_seq.h`` with the conventions of ``seq.py``: no fallback, nothing recorded by autograd,
``stream`` as there.  Tensors on another device than the current one make the call run on that device.  As a serving step
makes these calls for single tokens, their arguments are marshalled by a native module (``_seq_cache.so``).

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

from . import _check, _i64, _vp, Im2winError, load_library
from .seq import _elsewhere

__all__ = ["seq_rotary_frequencies", "seq_rotary_forward", "seq_rotary_backward", "seq_cache_write", "seq_cache_read",
           "seq_paged_attention_workspace_bytes", "seq_paged_attention_forward"]

_native = None


def _load():
    """The native module (which needs torch loaded first)."""
    global _native
    import torch  # noqa: F401
    lib = load_library()  # says what to do where nothing is built
    lib.seq_rotary_frequencies.restype = ctypes.c_int
    lib.seq_rotary_frequencies.argtypes = [_vp, _i64] + [ctypes.c_double] * 5
    try:
        from . import _seq_cache
    except ImportError as e:
        raise RuntimeError("_seq_cache.so is not built or does not fit this torch (%s); run "
                           "`python -c 'import __graft_entry__ as g; g.build()'`" % e) from e
    _seq_cache.set_error(Im2winError)
    _native = _seq_cache
    return _native


def seq_rotary_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, trained: float = 0.0, low: float = 1.0,
                           high: float = 32.0):
    """Frequencies [rot/2] (host, fp64) of pairs of channels: base ** (-2i/rot),
    for contexts ``factor`` times as long as the ``trained`` one slowed down by
    ``factor`` where a pair turns at most ``low`` times within it, kept where it
    turns at least ``high`` times, on a straight line between; trained 0: all
    slowed down."""
    import torch
    _native or _load()
    freq = torch.empty(rot // 2 if rot > 1 else 1, dtype=torch.float64)
    _check(load_library().seq_rotary_frequencies(freq.data_ptr(), rot, base, factor, trained, low, high),
           "seq_rotary_frequencies")
    return freq


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
    return (_native or _load()).rotary(x, freq, positions, interleaved, amplitude, out, False)


def seq_rotary_backward(dy, freq, positions=None, interleaved: bool = False, amplitude: float = 1.0, out=None, stream=None):
    """The gradient of ``seq_rotary_forward``'s input from that of its result."""
    if stream is not None:
        return _elsewhere(stream, seq_rotary_backward, dy, freq, positions, interleaved, amplitude, out)
    return (_native or _load()).rotary(dy, freq, positions, interleaved, amplitude, out, True)


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
    return (_native or _load()).cache_write(k, v, k_pages, v_pages, table, start, count, k_scale, v_scale)


def seq_cache_read(k_pages, v_pages, table, length, L: int, dtype=None, k_scale=None, v_scale=None, k=None, v=None,
                   stream=None):
    """The first length[b] tokens of each sequence as dense (k, v), each
    [B][L][Hkv][D] of type ``dtype`` (that of the pages; fp32 for 8-bit ones),
    written to ``k`` and ``v`` where given; rows from length[b] on are zeros."""
    if stream is not None:
        return _elsewhere(stream, seq_cache_read, k_pages, v_pages, table, length, L, dtype, k_scale, v_scale, k, v)
    return (_native or _load()).cache_read(k_pages, v_pages, table, length, L, dtype, k_scale, v_scale, k, v)


def seq_paged_attention_workspace_bytes(q, k_pages, v_pages, table, k_scale=None, v_scale=None) -> int:
    """Bytes of workspace of ``seq_paged_attention_forward`` with these operands."""
    return (_native or _load()).paged_workspace_bytes(q, k_pages, v_pages, table, k_scale, v_scale)


def seq_paged_attention_forward(q, k_pages, v_pages, table, length, scale=None, cap: float = 0.0, bias=None, k_scale=None,
                                v_scale=None, out=None, ws=None, stream=None):
    """Attention of one new token of each sequence, q [B][H][D] (any strides,
    the last dimension dense), the last of its length[b] tokens, over the pages.
    Returns (out like q, lse [B][H] fp32); scale, cap and bias as in
    ``seq_attention_forward``, pages and table as in ``seq_cache_write``."""
    if stream is not None:
        return _elsewhere(stream, seq_paged_attention_forward, q, k_pages, v_pages, table, length, scale, cap, bias,
                          k_scale, v_scale, out, ws)
    return (_native or _load()).paged_attention(q, k_pages, v_pages, table, length, scale, cap, bias, k_scale, v_scale, out,
                                                ws)
