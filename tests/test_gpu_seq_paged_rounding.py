"""Attention over 16-bit pages whose values nearly cancel: the weights are held to more bits than the result."""
import pytest
import torch

import paper_2608_20725_amd as pkg
from gpu_util import say
from seq_cache_ref import Cache
from seq_ref import TINY, U, Attention, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,wide", [(8, None), (100, None), (100, 500)])
@pytest.mark.parametrize("D,G", [(64, 2), (128, 5), (72, 20), (32, 3)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_values_that_nearly_cancel(dt, D, G, n, wide):
    """Values of neighbouring tokens are each other's negative, so that the result is far below them.

    Bound: a weight in two terms of the type is off by u twice, u^2 of it (fp16's subnormals by 2^-39 of the row's
    largest: 2^-25 of 2^14), fp32 arithmetic by 2*e (see Attention), and only the result is rounded once to u."""
    say("cancel", dt, D, G, n, wide)
    c = Cache([n, n - 2], 16, 2, D, dt, wide=wide)
    c.v[:, 1::2] = -c.v[:, 0::2]
    c._fill(c.v_pages, c.v.to(dt))
    q = (torch.randn((2, 2 * G, D), generator=torch.Generator().manual_seed(n)) * 2.0 ** -5).to(dt)
    ref = Attention(q[:, None], c.k, c.v, causal=True, align_end=True, kv_len=c.len)
    u, size = U[dt], (ref.p @ ref.v.abs())
    err = (u * u + 2 * ref.e) * size + 2.0 ** -38 * ref.v.abs().sum(2, keepdim=True)
    tol = u * (ref.out.abs() + err) + err + TINY[dt]
    kp, vp, table, _ = c.device()
    got, _ = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda())
    check(got, ref.out[:, :, 0], tol[:, :, 0], "out")
