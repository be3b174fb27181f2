"""Attention over pages of large batches: sequences without keys, with one and with many parts beside each other, in
several groups of the 64 that a wave scans at once, joined by one workgroup a row and by one for eight rows."""
import pytest
import torch

import paper_2608_20725_amd as pkg
from gpu_util import say
from seq_cache_ref import E4M3, Cache, attention
from seq_ref import check

pytestmark = pytest.mark.gpu

F32, F16, BF16, I8 = torch.float32, torch.float16, torch.bfloat16, torch.int8

# Sequences, key/value heads, queries each, channels, type, pages' type, whether keys are split: up to 512 sequences and
# 16383 pairs of a sequence and a tile of its heads.
BATCHES = [(65, 1, 1, 8, F32, F32, True), (129, 8, 3, 8, F16, F16, True), (129, 8, 3, 8, BF16, I8, True), (150, 2, 1, 8, F16, E4M3, True),
           (512, 1, 1, 8, BF16, BF16, True), (512, 4, 2, 8, F16, I8, True), (513, 1, 1, 8, BF16, BF16, False),
           (513, 4, 2, 8, F16, I8, False), (255, 64, 1, 8, F16, F16, True), (257, 64, 1, 8, F16, F16, False),
           (130, 4, 2, 64, BF16, BF16, True), (130, 4, 2, 64, F16, I8, True), (70, 1, 65, 16, F32, I8, True),
           (200, 2, 17, 40, BF16, E4M3, True)]


@pytest.mark.parametrize("case", BATCHES, ids=lambda c: "%dx%dx%d-%d-%s-%s" % (*c[:4], str(c[4])[6:], str(c[5])[6:]))
def test_batches(case):
    B, Hkv, G, D, dt, ct, split = case
    say("batch", case)
    g = torch.Generator().manual_seed(B + D)
    for k in range(2):
        # 0, 1, some and many tokens beside each other; the second time also 63 empty sequences in a row
        lens = torch.randint(0, 60, (B,), generator=g)
        lens[1::5], lens[3::7], lens[2::11], lens[4::13] = 0, 1, 1100, 700
        if k:
            lens[1:64], lens[0], lens[-1] = 0, 1050, 999
        c = Cache(lens.tolist(), 16, Hkv, D, dt, ct, wide=200, heads_first=k == 1 and Hkv > 1)
        q = torch.randn((B, Hkv * G, D), generator=g).to(dt)
        out, lse, tol, tl = attention(q, c)
        kp, vp, table, scales = c.device()
        need = pkg.seq_paged_attention_workspace_bytes(q.cuda(), kp, vp, table, **scales)
        assert (need > 0) == split
        # a workspace and a result that hold something else before
        ws = torch.full((max(need, 16) // 4,), float("nan"), device="cuda")
        got = torch.full((B, Hkv * G, D), float("nan"), dtype=dt, device="cuda")
        _, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), out=got, ws=ws, **scales)
        check(got, out, tol + 1e-30, "out")
        check(gl, lse, tl + 1e-30, "lse")
        empty = lens == 0
        assert not got[empty.cuda()].any() and torch.isneginf(gl[empty.cuda()]).all()
