"""Argument checks of the sequence operators with real device buffers: each
bad call is refused with its status before anything is launched."""
import pytest
import torch

import paper_2608_20725_amd as pkg

pytestmark = pytest.mark.gpu

EALIGN, EWORKSPACE, EOVERLAP, EBUFFER = -2, -6, -7, -8


def status(fn, *a, **k):
    with pytest.raises(pkg.Im2winError) as e:
        fn(*a, **k)
    return e.value.status


def test_attention():
    q = torch.zeros((2, 40, 4, 64), dtype=torch.float16, device="cuda")
    k = torch.zeros((2, 40, 2, 64), dtype=torch.float16, device="cuda")
    f = pkg.seq_attention_forward
    assert status(f, q, k, k, out=q) == EOVERLAP
    both = torch.zeros((2, 41, 4, 64), dtype=torch.float16, device="cuda")
    assert status(f, both[:, :40], k, k, out=both[:, 1:]) == EOVERLAP
    assert status(f, q, k, k, out=q[:, :, :1].expand(2, 40, 4, 64)) == EOVERLAP       # an output onto itself
    odd = torch.zeros(2 * 40 * 4 * 64 + 8, dtype=torch.float16, device="cuda")[4:4 + 2 * 40 * 4 * 64].view(2, 40, 4, 64)
    assert status(f, odd, k, k) == EALIGN
    wide = torch.zeros((2, 40, 4, 68), dtype=torch.float16, device="cuda")[..., :64]
    assert status(f, wide, k, k) == EALIGN
    out, lse = f(q, k, k)
    back = pkg.seq_attention_backward
    need = pkg.seq_attention_workspace_bytes(q, k, k, backward=True)
    assert need > 0
    assert status(back, q, q, k, k, out, lse, ws=torch.zeros(need - 16, dtype=torch.uint8, device="cuda")) == EWORKSPACE
    assert status(back, q, q, k, k, out, lse, dq=q) == EOVERLAP
    d = torch.empty_like(k)
    assert status(back, q, q, k, k, out, lse, dk=d, dv=d) == EOVERLAP
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    back(q, q, k, k, out, lse, ws=ws)
    host = [t.cpu() for t in (q, k, k)]
    assert status(f, *host) == EBUFFER


def test_layer_norm_and_bias():
    x = torch.zeros((6, 40), device="cuda")
    w = torch.zeros(40, device="cuda")
    f = pkg.seq_layer_norm_forward
    flat = torch.zeros(7 * 40, device="cuda")
    assert status(f, flat[:240].view(6, 40), w, w, out=flat[40:].view(6, 40)) == EOVERLAP
    wide = torch.zeros((6, 80), device="cuda")
    assert status(f, wide[:, :40], w, w, out=wide.view(-1)[:240].view(6, 40)) == EOVERLAP   # in place needs dense rows
    y, mean, rstd = f(x, w, w)
    need = pkg.seq_layer_norm_workspace_bytes(6, 40)
    ws = torch.zeros(need - 16, dtype=torch.uint8, device="cuda")
    assert status(pkg.seq_layer_norm_backward, x, x, w, mean, rstd, ws=ws) == EWORKSPACE
    assert status(f, x.cpu(), w.cpu(), w.cpu()) == EBUFFER
    table = torch.zeros((32, 4), device="cuda")
    big = torch.zeros(4 * 257 + 128, device="cuda")
    t = big[:128].view(32, 4)
    assert status(pkg.seq_rel_bias_forward, t, 128, out=big[64:64 + 4 * 257].view(4, 257)) == EOVERLAP
    assert status(pkg.seq_rel_bias_forward, table.cpu(), 128) == EBUFFER
