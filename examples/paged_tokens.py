"""An attention block with rotary positions: training, then serving over pages.

    python examples/paged_tokens.py [steps]

The block turns queries and keys by their tokens' positions and is trained on
smooth sequences of features to predict the next token's.  Then it serves
prompts of different lengths out of one pool of pages: the prompts arrive in
pieces (turn, write into the pages, read back what is there, attend), the
following tokens one by one (turn, write, attend over the pages), once with
pages of the block's own type and once in 8 bits, a quarter of fp32's bytes.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_20725_amd as im2win  # noqa: E402


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, freq):
        ctx.freq = freq
        return im2win.seq_rotary_forward(x, freq)

    @staticmethod
    def backward(ctx, dy):
        return im2win.seq_rotary_backward(dy.contiguous(), ctx.freq), None


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v):
        out, lse = im2win.seq_attention_forward(q, k, v, causal=True)
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    def backward(ctx, dout):
        return im2win.seq_attention_backward(dout.contiguous(), *ctx.saved_tensors, causal=True)[:3]


class Block(torch.nn.Module):
    """x + W_o attention(turned W_qk x, W_v x), then a linear head; H query heads over Hkv key/value heads."""

    def __init__(self, C=128, H=4, Hkv=2, dtype=torch.float32):
        super().__init__()
        self.H, self.Hkv, self.D = H, Hkv, C // H
        self.qkv = torch.nn.Linear(C, (H + 2 * Hkv) * self.D, dtype=dtype)
        self.out, self.head = torch.nn.Linear(C, C, dtype=dtype), torch.nn.Linear(C, C, dtype=dtype)
        self.freq = im2win.seq_rotary_frequencies(self.D)

    def project(self, x):
        """(queries and keys side by side, values)."""
        y = self.qkv(x).view(*x.shape[:2], self.H + 2 * self.Hkv, self.D)
        return y[:, :, :self.H + self.Hkv], y[:, :, self.H + self.Hkv:]

    def finish(self, x, a):
        return self.head(x + self.out(a.reshape(x.shape)))

    def forward(self, x):
        qk, v = self.project(x)
        qk = Rotary.apply(qk, self.freq)
        return self.finish(x, Attention.apply(qk[:, :, :self.H], qk[:, :, self.H:], v))


class Server:
    """A block's cache: one pool of pages for all its sequences."""

    def __init__(self, block, pages, page, table, kind):
        dev, shape = block.head.weight.device, (pages, page, block.Hkv, block.D)
        self.block, self.table, self.kind = block, table, kind
        self.k, self.v = torch.zeros(shape, dtype=kind, device=dev), torch.zeros(shape, dtype=kind, device=dev)
        self.scales = {}
        if kind in (torch.int8, torch.float8_e4m3fn):
            self.scales = {n: torch.zeros(shape[:3], device=dev) for n in ("k_scale", "v_scale")}
        self.len = torch.zeros(table.shape[0], dtype=torch.int32, device=dev)

    @torch.no_grad()
    def step(self, x, count=None):
        """The block's results for the next tokens x [B][n][C], of which count[b] are of sequence b (all n by default)."""
        b = self.block
        qk, v = b.project(x)
        qk = im2win.seq_rotary_forward(qk, b.freq, self.len)
        k = qk[:, :, b.H:]
        im2win.seq_cache_write(k, v, self.k, self.v, self.table, self.len, count, **self.scales)
        new = self.len + (x.shape[1] if count is None else count)
        if x.shape[1] == 1 and count is None:
            a, _ = im2win.seq_paged_attention_forward(qk[:, 0, :b.H], self.k, self.v, self.table, new, **self.scales)
        else:
            longest = int(new.max())
            k, v = im2win.seq_cache_read(self.k, self.v, self.table, new, longest, dtype=x.dtype, **self.scales)
            # queries of the piece see the sequence up to themselves: its first new token is at position len
            a = torch.empty_like(x).view(*x.shape[:2], b.H, b.D)
            for i in range(x.shape[0]):  # pieces of different starts: a call each
                n = int(new[i] - self.len[i])
                if n:
                    im2win.seq_attention_forward(qk[i:i + 1, :n, :b.H], k[i:i + 1], v[i:i + 1], causal=True, align_end=True,
                                                 kv_len=new[i:i + 1], out=a[i:i + 1, :n])
        self.len = new
        return b.finish(x, a)


def serve(block, x, prompts, piece, page, kind):
    """Results of every token of x [B][L][C]: the first prompts[b] in pieces, the others one by one."""
    B, L, _ = x.shape
    each = (L + page - 1) // page
    table = torch.randperm(B * each, device=x.device).int().view(B, each)
    server = Server(block, B * each, page, table, kind)
    out = torch.zeros_like(x)
    done = [0] * B
    while any(d < p for d, p in zip(done, prompts)):
        n = [min(piece, p - d) for d, p in zip(done, prompts)]
        part = torch.zeros((B, max(n), x.shape[2]), dtype=x.dtype, device=x.device)
        for b in range(B):
            part[b, :n[b]] = x[b, done[b]:done[b] + n[b]]
        y = server.step(part, torch.tensor(n, dtype=torch.int32, device=x.device))
        for b in range(B):
            out[b, done[b]:done[b] + n[b]] = y[b, :n[b]]
            done[b] += n[b]
    for _ in range(L - max(prompts)):  # one token of every sequence a step
        part = torch.stack([x[b, done[b]:done[b] + 1] for b in range(B)])
        y = server.step(part)
        for b in range(B):
            out[b, done[b]] = y[b, 0]
            done[b] += 1
    return out, done


def main(steps=20):
    torch.manual_seed(0)
    dev = torch.device("cuda")
    t = torch.arange(96, device=dev)[None, :, None] / 96
    w = torch.randn(8, 1, 128, device=dev) * 6
    x = torch.sin(t * w + torch.randn(8, 1, 128, device=dev))
    block = Block().to(dev)
    opt = torch.optim.Adam(block.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        loss = (block(x)[:, :-1] - x[:, 1:]).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    with torch.no_grad():
        whole = block(x)
    off = {}
    for kind in (torch.float32, torch.int8, torch.float8_e4m3fn):
        got, done = serve(block, x, prompts=[40, 64, 1, 33, 64, 17, 50, 2], piece=24, page=16, kind=kind)
        seen = torch.zeros_like(whole)
        for b, n in enumerate(done):
            seen[b, :n] = whole[b, :n]
        off[kind] = float((got - seen).norm() / seen.norm())
    print("loss %.4f -> %.4f over %d steps; served against whole: %s" % (
        losses[0], losses[-1], steps, ", ".join("%s %.2g" % (str(k)[6:], v) for k, v in off.items())), flush=True)
    return losses, off


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
