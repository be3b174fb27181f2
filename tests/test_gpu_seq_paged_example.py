"""The rotary operators and the paged cache as the example uses them: gradients
of its training step, and serving that gives what the whole call gives."""
import copy
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_tokens.py")


def load():
    spec = importlib.util.spec_from_file_location("paged_tokens", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_example():
    losses, off = load().main(steps=5)
    assert all(torch.isfinite(torch.tensor(losses)))
    # fp32 pages: the same sums in another order, through attention and two linear maps
    assert off[torch.float32] < 2e-5
    # int8: each key and value is off by at most half a step, 1/254 of its head's largest, e4m3 by 2^-4 of itself;
    # the block adds its input, so its result moves by less than the attention's share
    assert off[torch.int8] < 1 / 254 * 4 and off[torch.float8_e4m3fn] < 2.0 ** -4 * 2


def test_gradients_match_plain_autograd():
    """One step's parameter gradients against the same block in plain fp64."""
    ex = load()
    torch.manual_seed(1)
    block = ex.Block(C=64, H=4, Hkv=2).cuda()
    x = torch.randn(2, 50, 64, device="cuda")
    block(x).square().mean().backward()
    p = {n: t.detach().double().requires_grad_() for n, t in copy.deepcopy(block).named_parameters()}
    X = x.double()
    y = (X @ p["qkv.weight"].t() + p["qkv.bias"]).view(2, 50, 8, 16)
    t = torch.arange(50, device="cuda", dtype=torch.float64)[:, None] * block.freq.cuda()
    c, s = t.cos()[None, :, None], t.sin()[None, :, None]
    a, b = y[:, :, :6, :8], y[:, :, :6, 8:]
    qk = torch.cat([a * c - b * s, a * s + b * c], -1)
    q, k, v = qk[:, :, :4], qk[:, :, 4:].repeat_interleave(2, 2), y[:, :, 6:].repeat_interleave(2, 2)
    z = torch.einsum("bihd,bjhd->bhij", q, k) / 4
    z = z.masked_fill(torch.ones(50, 50, device="cuda").triu(1).bool(), float("-inf"))
    o = torch.einsum("bhij,bjhd->bihd", z.softmax(-1), v).reshape(2, 50, 64)
    out = (X + o @ p["out.weight"].t() + p["out.bias"]) @ p["head.weight"].t() + p["head.bias"]
    out.square().mean().backward()
    # fp32 sums of up to a few thousand terms, chained five deep
    for n, g in block.named_parameters():
        err = float((g.grad.double() - p[n].grad).norm() / p[n].grad.norm())
        assert err < 2e-5, (n, err)
