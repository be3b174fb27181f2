"""Plain implementations in 64 bits, on the CPU, of rotary positions, the paged
cache and its 8-bit numbers, and the error bounds of the kernels' arithmetic."""
from __future__ import annotations

import math

import numpy as np
import torch

from seq_ref import TINY, U, Attention

E4M3 = torch.float8_e4m3fn


def frequencies(rot, base=10000.0, factor=1.0, trained=0.0, low=1.0, high=32.0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        w = min(1.0, max(0.0, (trained * f / (2 * math.pi) - low) / (high - low))) if trained else 0.0
        out.append(w * f + (1 - w) * f / factor)
    return out


def rotary(x, freq, positions, interleaved=False, amplitude=1.0, backward=False):
    """(y, tolerance).  Angles are reduced in long double (64-bit fractions), so
    that far positions are exact here too.

    Bound: the kernel's angle is off by the truncation to 2^-32 turns (1.5e-9
    radians) and three roundings of at most pi/4 (the residue, 2 pi 2^-32 and
    their product: 3 * 0.79 * 2^-24), its sine and cosine by another two
    roundings of values up to 1 and 2e-9 left out: together below 5 * 2^-24.
    The products with the amplitude, the two products and the sum add at most 4
    roundings, the result one of its type."""
    h = len(freq)
    f = np.array([np.longdouble(v) for v in freq])
    turns = positions.numpy().astype(np.longdouble)[..., None] * f / (2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
    t = (turns - np.floor(turns)).astype(np.float64) * (2 * math.pi)
    c, s = torch.from_numpy(np.cos(t))[:, :, None] * amplitude, torch.from_numpy(np.sin(t))[:, :, None] * amplitude
    if backward:
        s = -s
    xd = x.double()
    a, b = (xd[..., 0:2 * h:2], xd[..., 1:2 * h:2]) if interleaved else (xd[..., :h], xd[..., h:2 * h])
    y, tol = xd.clone(), torch.zeros_like(xd)
    p, q = a * c - b * s, a * s + b * c
    e = 9 * 2.0 ** -24 * abs(amplitude) * (a.abs() + b.abs()) + TINY[x.dtype] + 1e-40
    u = U[x.dtype]
    parts = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    for part, v in zip(parts, (p, q)):
        y[..., part] = v
        tol[..., part] = e + u * v.abs()
    return y, tol


def coded(x, ct):
    """(codes as numbers, fp32 scales) of x [..][D]."""
    top = x.double().abs().amax(-1)
    if ct == torch.int8:
        scale = (top.float() / torch.full_like(top, 127, dtype=torch.float32)).clamp(min=2.0 ** -126)
        scale = scale.clamp(max=float.fromhex("0x1.020406p+121"))  # the largest whose 127-fold is finite in fp32
        codes = torch.round(x.double() / scale.double()[..., None]).clamp(-127, 127)
    else:
        e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448))
        # log2 may be off next to a power of two
        e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)
        e = torch.where(top > 448 * torch.exp2(e), e + 1, e).clamp(min=-126)
        scale = torch.exp2(e).float()
        v = x.double() / scale.double()[..., None]
        place = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -40))).clamp(min=-6) - 3
        codes = torch.round(v * torch.exp2(-place)) * torch.exp2(place)
    broken = ~torch.isfinite(top)
    scale = torch.where(broken, torch.full_like(scale, float("nan")), scale)
    return codes, scale


class Cache:
    """Sequences of random tokens in shuffled pages; what no sequence holds is
    poisoned.  ``k``, ``v`` [B][longest][Hkv][D]: the values that the pages stand
    for, in 64 bits."""

    def __init__(self, lens, page, Hkv, D, dt, ct=None, heads_first=False, spare=2, wide=None, seed=0, size=1.0):
        g = torch.Generator().manual_seed(seed)
        self.ct, self.page, self.lens = ct or dt, page, lens
        need = [(n + page - 1) // page for n in lens]
        pages = sum(need) + spare
        wide = max(need + [1]) if wide is None else wide
        order = torch.randperm(max(pages, 1), generator=g).int()
        self.table = torch.full((len(lens), wide), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.len = torch.tensor(lens, dtype=torch.int32)
        longest = max(lens + [1])
        for name in ("k", "v"):
            x = torch.randn((len(lens), longest, Hkv, D), generator=g, dtype=torch.float64)
            x = (x * size * (0.25 + 2 * torch.rand((len(lens), longest, Hkv, 1), generator=g, dtype=torch.float64))).to(dt)
            if self.ct == dt:
                pool = torch.full((pages, page, Hkv, D), float("nan"), dtype=dt)
                self._fill(pool, x)
                scale, values = None, x.double()
            else:
                codes, s = coded(x, self.ct)
                pool = torch.randint(-100, 100, (pages, page, Hkv, D), generator=g).to(torch.int8)
                pool = pool if self.ct == torch.int8 else pool.view(E4M3)
                scale = torch.full((pages, page, Hkv), float("nan"))
                self._fill(pool, codes.to(self.ct))
                self._fill(scale, s)
                values = codes * s.double()[..., None]
                setattr(self, name + "_top", float(s.max()) if s.numel() else 0.0)
                setattr(self, name + "_codes", codes)
            if heads_first:
                pool = pool.transpose(1, 2).contiguous().transpose(1, 2)
                scale = None if scale is None else scale.transpose(1, 2).contiguous().transpose(1, 2)
            setattr(self, name, values)
            setattr(self, name + "_pages", pool)
            setattr(self, name + "_scale", scale)

    def _fill(self, pool, x):
        raw = pool.view(torch.uint8) if pool.dtype == E4M3 else pool
        src = x.view(torch.uint8) if x.dtype == E4M3 else x
        for b, n in enumerate(self.lens):
            for i in range((n + self.page - 1) // self.page):
                m = min(self.page, n - i * self.page)
                raw[int(self.table[b, i]), :m] = src[b, i * self.page:i * self.page + m]

    def device(self):
        """(k_pages, v_pages, table, scales) on the GPU, strides kept."""
        scales = {}
        if self.k_scale is not None:
            scales = {"k_scale": moved(self.k_scale), "v_scale": moved(self.v_scale)}
        return moved(self.k_pages), moved(self.v_pages), self.table.cuda(), scales


def moved(t):
    """A copy on the GPU with the strides of ``t``."""
    if t.is_contiguous():
        return t.cuda()
    return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)


def attention(q, cache, there=None, **opts):
    """(out, lse, tolerances) of one token a sequence.  ``there`` [B][longest]:
    tokens whose pages exist.

    Beyond seq_ref's bound: a value's weight P*s is rounded relative to the
    largest scale S (over at most 2*S as a power of two): fp16 subnormals are
    2^-39 of it, on codes instead of values."""
    dt = q.dtype
    B, L = cache.k.shape[:2]
    docs = {}
    if there is not None:
        docs = {"q_doc": torch.zeros((B, 1), dtype=torch.int32), "k_doc": torch.where(there, 0, -1).int()}
    ref = Attention(q[:, None], cache.k, cache.v, causal=True, align_end=True, kv_len=cache.len, **docs, **opts)
    ref.dtype = dt
    tol, tl = ref.tolerances()
    if cache.ct != dt:
        seen = (torch.arange(L)[None, :] < cache.len[:, None]).double()[:, :, None, None]
        codes = (cache.v_codes.abs() * seen).sum(1).repeat_interleave(ref.G, 1)
        tol = tol + (2.0 ** -38 * cache.v_top * codes)[:, None]
    return ref.out.transpose(1, 2)[:, 0], ref.lse[..., 0], tol[:, 0], tl[..., 0]
