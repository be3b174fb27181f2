"""Plain implementations of the sequence operators in 64 bits, on the CPU, and
the error bounds of the kernels' arithmetic.

u is the unit roundoff of the element type (fp16 2^-11, bf16 2^-8), 0 for the
intermediate roundings that fp32 does not have."""
from __future__ import annotations

import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# a result below the smallest normal number is off by half the spacing there
# (fp16: 2^-14 and 2^-24; below 2^-126 nothing here lies)
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
U_INNER = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def bucket(d, buckets, R, two_sided):
    d = max(-R, min(R, d))
    m, first = (buckets // 2, buckets // 2 if d > 0 else 0) if two_sided else (buckets, 0)
    n, e = abs(d) if two_sided else max(0, -d), (buckets // 2 if two_sided else buckets) // 2
    if n < e:
        return first + n
    return first + min(m - 1, math.floor(e + (m - e) * math.log(n / e) / math.log(R / e) + 1e-9))


def allowed(B, Lq, Lk, causal=False, align_end=False, kv_len=None, prefix=None, q_doc=None, k_doc=None):
    """([B][Lq][Lk] pairs that take part, [B][Lq][Lk] key minus query position)"""
    oks, ds = [], []
    for b in range(B):
        n = Lk if kv_len is None else max(0, min(Lk, int(kv_len[b])))
        i, j = torch.arange(Lq)[:, None], torch.arange(Lk)[None, :]
        p = i + (n - Lq if align_end else 0)
        ok = (j < n) & (p == p)
        if causal:
            see = j <= p
            if prefix is not None:
                see = see | (j < int(prefix[b]))
            ok = ok & see
        if q_doc is not None:
            ok = ok & (q_doc[b][:, None] == k_doc[b][None, :]) & (q_doc[b][:, None] >= 0)
        oks.append(ok)
        ds.append(j - p)
    return torch.stack(oks), torch.stack(ds)


class Attention:
    """Attention of the given (rounded) inputs; left-out pairs have no part, so
    what they hold is replaced before any arithmetic."""

    def __init__(self, q, k, v, scale=None, cap=0.0, bias=None, **masks):
        self.dtype = q.dtype
        B, Lq, H, D = q.shape
        Lk, Hk = k.shape[1], k.shape[2]
        self.G, self.scale, self.cap = H // Hk, D ** -0.5 if scale is None else scale, cap
        self.q = q.double().transpose(1, 2)
        self.k = k.double().transpose(1, 2).repeat_interleave(self.G, 1)
        self.v = v.double().transpose(1, 2).repeat_interleave(self.G, 1)
        ok, d = allowed(B, Lq, Lk, **masks)
        self.ok = ok[:, None].expand(B, H, Lq, Lk)
        x = (self.q @ self.k.transpose(2, 3)) * self.scale
        self.t = torch.tanh(x / cap) if cap else None
        s = cap * self.t if cap else x
        self.R, self.d = 0, None
        if bias is not None:
            self.R = bias.shape[1] // 2
            self.d = d.clamp(-self.R, self.R) + self.R
            s = s + bias.double()[:, self.d].transpose(0, 1)
        s = torch.where(self.ok, s, torch.full_like(s, -math.inf))
        self.lse = torch.logsumexp(s, -1)
        z = torch.where(torch.isinf(self.lse), torch.zeros_like(self.lse), self.lse)[..., None]
        self.p = torch.where(self.ok, (s - z).exp(), torch.zeros_like(s))
        self.out = self.p @ self.v
        # fp32 arithmetic: a score's error is at most 2^-24 (D+4) sum|q||k|
        # scale, plus a few roundings of values up to |s| and |lse|; as
        # probabilities are exponentials, their relative error is that of
        # s - lse; Lk + 64 more roundings cover the sums
        sa = float((self.q.abs() @ self.k.abs().transpose(2, 3)).max()) * self.scale if Lk and Lq and B else 0.0
        big = sa + (float(bias.abs().max()) if bias is not None else 0.0)
        fin = self.lse[torch.isfinite(self.lse)]
        big += float(fin.abs().max()) if fin.numel() else 0.0
        self.e = 2.0 ** -24 * (2 * (D + 4) * sa + 8 * big + cap * 4 + Lk + 64)

    def tolerances(self):
        """(out, lse): 16-bit rounds P (relative u; fp16 also 2^-39 of the
        row's largest, its subnormals) and the result."""
        u, ui = U[self.dtype], U_INNER[self.dtype]
        a = self.p @ self.v.abs()
        out = (u + ui + 2 * self.e) * a + 2.0 ** -38 * self.v.abs().sum(2, keepdim=True) + TINY[self.dtype]
        return out.transpose(1, 2), torch.full_like(self.lse, self.e) + 2.0 ** -22 * self.lse.abs().nan_to_num(posinf=0)

    def grads(self, dout, out, lse):
        """(dq, dk, dv, dstrip) and their tolerances, from dout and the
        forward results the call was given."""
        do, o = dout.double().transpose(1, 2), out.double().transpose(1, 2)
        l = lse.double()[..., None]
        s = self.p  # recompute from the given lse: s - lse
        fin = torch.isfinite(l) & self.ok
        p = torch.where(fin, s * (torch.where(torch.isinf(self.lse), torch.zeros_like(self.lse), self.lse)[..., None]
                                  - torch.where(torch.isinf(l), torch.zeros_like(l), l)).exp(), torch.zeros_like(s))
        dp, delta = do @ self.v.transpose(2, 3), (do * o).sum(-1, keepdim=True)
        ds = p * torch.where(self.ok, dp - delta, torch.zeros_like(dp))
        size = p * (do.abs() @ self.v.abs().transpose(2, 3) + (do * o).abs().sum(-1, keepdim=True))  # of the terms of ds
        slope = 1 - self.t ** 2 if self.cap else torch.ones_like(ds)
        dx = ds * slope * self.scale
        u, ui, e = U[self.dtype], U_INNER[self.dtype], self.e
        err = (2 * e + 2.0 ** -24 * self.q.shape[-1]) * size          # of ds
        # fp16 subnormals of the scaled gradients: 2^-25 of a bound that is at
        # most 2^15 after scaling by at least half
        bound = 2 * float(do.norm(dim=-1).max()) * float(self.v.norm(dim=-1).max()) if do.numel() and self.v.numel() else 0
        tiny = bound * 2.0 ** -38 if self.dtype == torch.float16 else 0.0
        ex = (err + ui * ds.abs() + tiny) * self.scale                # of dx (slopes are at most 1, their error in e)
        dq, tq = dx @ self.k, ex @ self.k.abs()
        dk, tk = dx.transpose(2, 3) @ self.q, ex.transpose(2, 3) @ self.q.abs()
        dv, tv = p.transpose(2, 3) @ do, ((ui + 2 * e) * p + 2.0 ** -38).transpose(2, 3) @ do.abs()
        tq = tq + u * dq.abs() + TINY[self.dtype]
        B, H = dk.shape[:2]

        def group(x):
            return x.reshape(B, H // self.G, self.G, *x.shape[2:]).sum(2).transpose(1, 2)
        dk, tk, dv, tv = group(dk), group(tk), group(dv), group(tv)
        tk, tv = tk + u * dk.abs() + TINY[self.dtype], tv + u * dv.abs() + TINY[self.dtype]
        # sums of products in fp32
        n = 2.0 ** -24 * (max(ds.shape[2:]) + 64) if ds.numel() else 0.0
        tq = tq + n * (dx.abs() @ self.k.abs())
        tk = tk + n * group(dx.abs().transpose(2, 3) @ self.q.abs())
        dstrip = ts = None
        if self.R:
            dstrip = torch.zeros((H, 2 * self.R + 1), dtype=torch.float64)
            ts = torch.zeros_like(dstrip)
            for b in range(B):
                at = self.d[b].reshape(-1)
                dstrip.index_add_(1, at, ds[b].reshape(H, -1))
                ts.index_add_(1, at, (err + 2.0 ** -20 * ds.abs())[b].reshape(H, -1))
            ts = ts + 1e-30
        return (dq.transpose(1, 2), dk, dv, dstrip), (tq.transpose(1, 2) + 1e-30, tk + 1e-30, tv + 1e-30, ts)


def check(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    assert not torch.isnan(got).any(), "%s: NaN" % what
    same = (got == want)  # covers infinities
    over = (got - want).abs() / tol
    over = torch.where(same, torch.zeros_like(over), over)
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, "%s: error %.3g of the bound" % (what, worst)
    return worst
