"""A convolutional stem and an attention block over its pixels.

    python examples/conv_tokens.py [steps]

Images go through a frozen strided convolution (im2win_conv2d); its output
pixels are the tokens of one pre-norm attention block with a learned bias by
distance, which is trained to predict the next token's features in raster
order.  Then the trained block runs as a server would: a prompt in one call,
the following tokens one by one over a key/value cache, with the same results.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_20725_amd as im2win  # noqa: E402


class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        y, mean, rstd = im2win.seq_layer_norm_forward(x, weight, bias)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        return im2win.seq_layer_norm_backward(dy.contiguous(), *ctx.saved_tensors)


class RelBias(torch.autograd.Function):
    """Bucket table [buckets][H] -> strip by distance [H][2R+1]."""

    @staticmethod
    def forward(ctx, table, max_distance):
        ctx.buckets, ctx.dtype = table.shape[0], table.dtype
        return im2win.seq_rel_bias_forward(table, max_distance, two_sided=False)

    @staticmethod
    def backward(ctx, dstrip):
        return im2win.seq_rel_bias_backward(dstrip.contiguous(), ctx.buckets, two_sided=False, dtype=ctx.dtype), None


class Attention(torch.autograd.Function):
    """Causal attention of the columns of a packed [B][L][3][H][D] tensor."""

    @staticmethod
    def forward(ctx, qkv, strip):
        q, k, v = qkv.unbind(2)
        out, lse = im2win.seq_attention_forward(q, k, v, bias=strip, causal=True)
        ctx.save_for_backward(qkv, strip, out, lse)
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, strip, out, lse = ctx.saved_tensors
        q, k, v = qkv.unbind(2)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = dqkv.unbind(2)   # the gradients are written where the projection's backward reads them
        dstrip = im2win.seq_attention_backward(dout.contiguous(), q, k, v, out, lse, bias=strip, causal=True, dq=dq, dk=dk,
                                               dv=dv)[3]
        return dqkv, dstrip


class Block(torch.nn.Module):
    """x + W_o attention(W_qkv norm(x)), then a linear head."""

    def __init__(self, C=128, H=4, buckets=16, max_distance=64, dtype=torch.bfloat16):
        super().__init__()
        self.H, self.D, self.R = H, C // H, max_distance
        self.weight, self.bias = torch.nn.Parameter(torch.ones(C)), torch.nn.Parameter(torch.zeros(C))
        self.table = torch.nn.Parameter(torch.zeros(buckets, H))
        self.qkv, self.out, self.head = (torch.nn.Linear(C, n, dtype=dtype) for n in (3 * C, C, C))

    def project(self, x):
        h = LayerNorm.apply(x, self.weight, self.bias)
        return self.qkv(h).view(*x.shape[:2], 3, self.H, self.D)

    def finish(self, x, a):
        return self.head(x + self.out(a.reshape(x.shape)))

    def forward(self, x):
        return self.finish(x, Attention.apply(self.project(x), RelBias.apply(self.table, self.R)))

    @torch.no_grad()
    def serve(self, x, prompt):
        """The same results token by token: the first ``prompt`` tokens in one
        call, each later one against the cache."""
        B, L, C = x.shape
        strip = im2win.seq_rel_bias_forward(self.table, self.R, two_sided=False)
        cache_k = torch.empty((B, L, self.H, self.D), dtype=x.dtype, device=x.device)
        cache_v = torch.empty_like(cache_k)
        lens = torch.zeros(B, dtype=torch.int32, device=x.device)
        outs, at = [], 0
        for n in [prompt] + [1] * (L - prompt):
            part = x[:, at:at + n].contiguous()
            q, k, v = self.project(part).unbind(2)
            cache_k[:, at:at + n], cache_v[:, at:at + n] = k, v
            lens += n
            at += n
            a, _ = im2win.seq_attention_forward(q, cache_k, cache_v, bias=strip, causal=True, align_end=True, kv_len=lens)
            outs.append(self.finish(part, a))
        return torch.cat(outs, 1)


def tokens(images, filt, stride):
    """[N][H_o*W_o][C_o] features of NHWC images under a frozen convolution."""
    out, _ = im2win.im2win_conv2d(images, filt, stride)
    N, H, W, C = out.shape
    return out.view(N, H * W, C)


def main(steps=30):
    torch.manual_seed(0)
    dev = torch.device("cuda")
    filt = (torch.randn(4, 4, 3, 128, device=dev) / 7).to(torch.bfloat16)
    # smooth images: neighbouring pixels predict each other
    small = torch.randn(16, 3, 12, 12, device=dev)
    images = torch.nn.functional.interpolate(small, size=(64, 64), mode="bilinear")
    x = tokens(images.permute(0, 2, 3, 1).contiguous().to(torch.bfloat16), filt, 4)
    block = Block().to(dev)
    opt = torch.optim.Adam(block.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        loss = (block(x)[:, :-1].float() - x[:, 1:].float()).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    with torch.no_grad():
        whole = block(x)
    served = block.serve(x, prompt=200)
    diff = float((whole.float() - served.float()).norm() / whole.float().norm())
    print("loss %.4f -> %.4f over %d steps; served against whole: relative difference %.2g" % (
        losses[0], losses[-1], steps, diff), flush=True)
    return losses, diff


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
