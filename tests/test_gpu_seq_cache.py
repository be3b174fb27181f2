"""The paged cache: writing, reading back and attention over it, against plain
implementations in 64 bits."""
import pytest
import torch

import paper_2608_20725_amd as pkg
from gpu_util import say
from seq_cache_ref import E4M3, Cache, attention, coded, moved
from seq_ref import TINY, U, check

pytestmark = pytest.mark.gpu

F32, F16, BF16, I8 = torch.float32, torch.float16, torch.bfloat16, torch.int8
NAMES = {F32: "f32", F16: "f16", BF16: "bf16", I8: "i8", E4M3: "e4m3"}
PAIRS = [(F32, F32), (F16, F16), (BF16, BF16), (F32, I8), (F16, I8), (BF16, I8), (F32, E4M3), (F16, E4M3), (BF16, E4M3)]
ids = lambda v: "-".join(NAMES[t] for t in v) if isinstance(v[0], torch.dtype) else "".join(ch for ch in str(v) if ch in "0123456789,x")[:40]


def bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def same(got, want, what):
    n = int((bits(got.cpu()) != bits(want.cpu())).sum())
    assert n == 0, "%s: %d numbers differ" % (what, n)


def tokens(B, L, Hkv, D, dt, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, L, Hkv, D), generator=g, dtype=torch.float64)
    return (x * torch.exp2(torch.randint(-6, 7, (B, L, Hkv, 1), generator=g).double())).to(dt)


def poisoned(pages, page, Hkv, D, ct):
    if ct in (I8, E4M3):
        p = torch.full((pages, page, Hkv, D), 77, dtype=I8)
        return (p if ct == I8 else p.view(E4M3)), torch.full((pages, page, Hkv), 0.125)
    return torch.full((pages, page, Hkv, D), 7.0, dtype=ct), None


# heads, channels, page, tokens offered, (start, count) of each sequence
WRITES = [(2, 64, 16, 5, [(0, 5), (14, 4), (31, 0), (47, 1)]), (1, 8, 1, 9, [(0, 9), (2, 3)]),
          (3, 80, 24, 61, [(0, 61), (5, 50), (23, 25), (100, 1)]), (8, 128, 64, 130, [(0, 130), (63, 66), (1, 64)]),
          (2, 40, 7, 3, [(6, 3), (0, 1)]), (1, 128, 200, 1, [(199, 1), (200, 1), (0, 0)]), (5, 32, 33, 40, [(0, 40)])]


@pytest.mark.parametrize("heads_first", [False, True], ids=["tokens", "heads"])
@pytest.mark.parametrize("case", WRITES, ids=ids)
@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_write(types, case, heads_first):
    """Every number in its place and nothing else touched, bit for bit."""
    dt, ct = types
    Hkv, D, page, L, spans = case
    say("write", types, case, heads_first)
    B = len(spans)
    wide = max((s + n + page - 1) // page for s, n in spans) + 1
    table = torch.randperm(B * wide, generator=torch.Generator().manual_seed(3)).int().view(B, wide)
    k, v = tokens(B, L, Hkv, D, dt, 1), tokens(B, L, Hkv, D, dt, 2)
    k[0, 0, 0] = 0
    pools = [poisoned(B * wide + 1, page, Hkv, D, ct) for _ in range(2)]
    want = [(p.clone(), None if s is None else s.clone()) for p, s in pools]
    for (pool, scale), x in zip(want, (k, v)):
        codes, sc = (x, None) if scale is None else coded(x, ct)
        for b, (s, n) in enumerate(spans):
            for t in range(n):
                i, o = divmod(s + t, page)
                raw = pool.view(torch.uint8) if ct == E4M3 else pool
                raw[table[b, i], o] = codes[b, t].to(ct).view(torch.uint8) if ct == E4M3 else codes[b, t].to(ct)
                if sc is not None:
                    scale[table[b, i], o] = sc[b, t]
    if heads_first:
        pools = [(p.transpose(1, 2).contiguous().transpose(1, 2), None if s is None else s.transpose(1, 2).contiguous().transpose(1, 2))
                 for p, s in pools]
    (kp, ks), (vp, vs) = [(moved(p), None if s is None else moved(s)) for p, s in pools]
    scales = {} if ks is None else {"k_scale": ks, "v_scale": vs}
    kv = torch.stack([k, v], 2).cuda()  # side by side in each token's row
    start, count = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in zip(*spans))
    assert pkg.seq_cache_write(kv[:, :, 0], kv[:, :, 1], kp, vp, table.cuda(), start, count, **scales) is None
    for got, gs, (p, s) in ((kp, ks, want[0]), (vp, vs, want[1])):
        same(got, p, "codes")
        if s is not None:
            same(gs, s, "scales")


def test_write_without_start_and_count():
    k, v = tokens(2, 20, 2, 64, F16, 1).cuda(), tokens(2, 20, 2, 64, F16, 2).cuda()
    kp, vp = torch.zeros(4, 16, 2, 64, dtype=F16, device="cuda"), torch.zeros(4, 16, 2, 64, dtype=F16, device="cuda")
    table = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device="cuda")
    pkg.seq_cache_write(k, v, kp, vp, table)
    for x, p in ((k, kp), (v, vp)):
        for b in range(2):
            seq = p[table[b].long()].flatten(0, 1)
            assert torch.equal(seq[:20], x[b]) and not seq[20:].any()


@pytest.mark.parametrize("ct", [None, I8, E4M3])
def test_write_to_places_that_are_not_there(ct):
    """Positions before the first and behind the last page, and entries that
    name no page, take nothing; the other tokens are written."""
    k = tokens(3, 40, 2, 64, F32, 4)
    pool, scale = poisoned(5, 16, 2, 64, ct or F32)
    table = torch.tensor([[4, 0, 1], [-1, 2, 5], [3, -2 ** 31, 2 ** 31 - 1]], dtype=torch.int32)
    start = torch.tensor([-3, 8, 20], dtype=torch.int32)  # row 0: from -3 on; row 2: until 59 of 48
    want, ws = pool.clone(), None if scale is None else scale.clone()
    codes, sc = (k, None) if scale is None else coded(k, ct)
    raw = want.view(torch.uint8) if ct == E4M3 else want
    for b in range(3):
        for t in range(40):
            p = int(start[b]) + t
            if 0 <= p < 48 and 0 <= table[b, p // 16] < 5:
                raw[table[b, p // 16], p % 16] = codes[b, t].to(want.dtype).view(raw.dtype) if ct == E4M3 else codes[b, t].to(want.dtype)
                if sc is not None:
                    ws[table[b, p // 16], p % 16] = sc[b, t]
    kp, vp = pool.cuda(), pool.cuda()
    scales = {} if scale is None else {"k_scale": scale.cuda(), "v_scale": scale.cuda()}
    pkg.seq_cache_write(k.cuda(), k.cuda(), kp, vp, table.cuda(), start.cuda(), **scales)
    same(kp, want, "keys")
    same(vp, want, "values")
    for s in scales.values():
        same(s, ws, "scales")


@pytest.mark.parametrize("ct", [I8, E4M3], ids=["i8", "e4m3"])
def test_numbers_of_8_bits_at_their_borders(ct):
    """Halves between two codes, the largest and smallest magnitudes, zeros,
    scales at 2^-126, values that are not finite."""
    x = torch.zeros(1, 24, 1, 64)
    x[0, 0, 0] = torch.arange(64) - 31.5                           # ties of a scale of 0.25 (top 31.75 below)
    x[0, 0, 0, 0] = 31.75
    x[0, 1, 0, :] = torch.linspace(-127, 127, 64)
    x[0, 2, 0, :4] = torch.tensor([127.0, 0.5, 1.5, -2.5])         # scale 1: halves go to the even code
    x[0, 3, 0, :2] = torch.tensor([3.4028234663852886e38, -1e38])
    x[0, 4, 0, :3] = torch.tensor([1e-45, -3e-45, 1.2e-38])
    x[0, 5, 0, 0] = 2.0 ** -126
    x[0, 6, 0, 5] = -448.0
    x[0, 7, 0, 5] = 448.0000305
    x[0, 8, 0, :] = torch.exp2(torch.linspace(-20, 0, 64))
    x[0, 9, 0, :] = 1.0 + torch.arange(64) / 64 * 0.5              # ties of three fraction bits
    x[0, 10, 0, :] = (torch.arange(64) + 0.5) * 2.0 ** -10         # and of subnormal codes beside 448
    x[0, 10, 0, 63] = 448
    g = torch.Generator().manual_seed(5)
    x[0, 11:20, 0] = torch.randn(9, 64, generator=g) * torch.exp2(torch.randint(-120, 120, (9, 1), generator=g).float())
    x[0, 20, 0, 7], x[0, 21, 0, 8], x[0, 22, 0, 9] = float("nan"), float("inf"), -float("inf")
    x[0, 23, 0, 3] = 2.0 ** -149
    codes, s = coded(x, ct)
    kp, sp = poisoned(1, 24, 1, 64, ct)
    kp, vp, ks, vs = kp.cuda(), kp.cuda(), sp.cuda(), sp.cuda()
    table, n = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([24], dtype=torch.int32, device="cuda")
    pkg.seq_cache_write(x.cuda(), -x.cuda(), kp, vp, table, k_scale=ks, v_scale=vs)
    fine = torch.isfinite(s[0, :, 0])
    assert fine.sum() == 21
    for p, sc, sign in ((kp, ks, 1), (vp, vs, -1)):
        assert torch.equal(sc[0, fine, 0].cpu(), s[0, fine, 0]) and torch.isnan(sc[0, ~fine, 0]).all()
        assert torch.equal(p.float().double().cpu()[0, fine, 0], sign * codes[0, fine, 0])
    k, v = pkg.seq_cache_read(kp, vp, table, n, 24, k_scale=ks, v_scale=vs)
    assert torch.isnan(k[0, ~fine]).all() and torch.isnan(v[0, ~fine]).all()
    # the product is exact in 64 bits and rounded once to fp32 (e4m3's nearest
    # number to fp32's largest is 2^128: infinity)
    value = (codes * s.double()[..., None])[0, fine]
    assert torch.equal(k[0, fine].cpu(), value.float())
    assert torch.equal(v[0, fine], -k[0, fine])


# lengths, page, heads, channels, rows asked for
READS = [([0, 1, 15, 16, 17, 100], 16, 2, 64, 100), ([40, 3], 1, 1, 8, 50), ([61, 200, 0], 24, 3, 80, 90),
         ([130, 64, 65], 64, 8, 128, 130), ([9], 7, 2, 40, 3), ([300, 299], 200, 1, 32, 600)]


@pytest.mark.parametrize("case", READS, ids=ids)
@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_read(types, case):
    dt, ct = types
    lens, page, Hkv, D, L = case
    say("read", types, case)
    for heads_first in (False, True):
        c = Cache(lens, page, Hkv, D, dt, ct, heads_first)
        kp, vp, table, scales = c.device()
        both = torch.full((len(lens), L, 2, Hkv, D), float("nan"), dtype=dt, device="cuda")
        out = {} if heads_first else {"k": both[:, :, 0], "v": both[:, :, 1]}
        got = pkg.seq_cache_read(kp, vp, table, c.len.cuda(), L, dtype=dt, **scales, **out)
        for x, want in zip(got, (c.k, c.v)):
            for b, n in enumerate(lens):
                m = min(n, L)
                assert not x[b, n:].any(), "rows behind a sequence are zeros"
                if ct == dt:
                    assert torch.equal(x[b, :m].cpu().double(), want[b, :m])
                else:  # code * scale, a rounding in fp32 and one to the type
                    w = want[b, :m]
                    check(x[b, :m], w, (U[dt] + 2.0 ** -23) * w.abs() + TINY[dt] + 2.0 ** -149, "read")


def test_read_of_pages_that_are_not_there_and_shared_ones():
    c = Cache([40, 40], 16, 2, 64, F32)
    kp, vp, table, _ = c.device()
    table[1] = table[0]      # a shared prefix
    table[0, 1] = -1
    table[1, 2] = kp.shape[0]
    n = torch.tensor([40, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    k, v = pkg.seq_cache_read(kp, vp, table, n, 60)
    for x, want in ((k.cpu().double(), c.k), (v.cpu().double(), c.v)):
        assert torch.equal(x[0, :16], want[0, :16]) and not x[0, 16:32].any() and torch.equal(x[0, 32:40], want[0, 32:40])
        assert not x[0, 40:].any()
        assert torch.equal(x[1, :32], want[0, :32]) and not x[1, 32:].any()


# lengths, page, key/value heads, queries each, channels
ATTNS = [([1, 31, 32, 33, 0], 16, 2, 4, 64), ([127, 128, 129, 2500], 24, 1, 3, 80), ([1000], 64, 4, 8, 128),
         ([5, 257], 1, 2, 1, 8), ([640, 3], 200, 1, 17, 128), ([300], 5, 2, 40, 72), ([700, 90], 33, 1, 65, 96),
         ([129] * 40, 16, 2, 16, 40), ([4100, 1], 128, 1, 100, 64)]


@pytest.mark.parametrize("case", ATTNS, ids=ids)
@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_attention(types, case):
    dt, ct = types
    lens, page, Hkv, G, D = case
    say("paged", types, case)
    g = torch.Generator().manual_seed(11)
    for k, opts in enumerate(({}, {"cap": 20.0, "R": 50}, {"scale": 0.4, "R": 3})):
        c = Cache(lens, page, Hkv, D, dt, ct, heads_first=k == 1, seed=k)
        q = torch.randn((len(lens), Hkv * G, D), generator=g).to(dt)
        opts = dict(opts)
        R = opts.pop("R", 0)
        bias = torch.randn((Hkv * G, 2 * R + 1), generator=g) if R else None
        out, lse, tol, tl = attention(q, c, bias=bias, **opts)
        kp, vp, table, scales = c.device()
        got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(),
                                                  bias=None if bias is None else bias.cuda(), **scales, **opts)
        check(got, out, tol + 1e-30, "out %d" % k)
        check(gl, lse, tl + 1e-30, "lse %d" % k)


@pytest.mark.parametrize("D,G", [(64, 3), (128, 4), (72, 17), (128, 40), (40, 1)])
@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_a_table_far_longer_than_its_sequences(types, D, G):
    """Few keys and many parts wanted: parts without keys, one sequence beside
    empty ones; and the larger tiles, which a table of this width chooses."""
    dt, ct = types
    lens = [3, 0, 400, 129, 1301]
    g = torch.Generator().manual_seed(1)
    for heads_first in (False, True):
        c = Cache(lens, 16, 2, D, dt, ct, wide=2000, heads_first=heads_first)
        q = torch.randn((5, 2 * G, D), generator=g).to(dt)
        bias = torch.randn((2 * G, 2 * 60 + 1), generator=g) if heads_first else None
        cap = 25.0 if heads_first else 0.0
        out, lse, tol, tl = attention(q, c, bias=bias, cap=cap)
        kp, vp, table, scales = c.device()
        got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), cap=cap,
                                                  bias=None if bias is None else bias.cuda(), **scales)
        check(got, out, tol + 1e-30, "out")
        check(gl, lse, tl + 1e-30, "lse")
        assert not got[1].any() and torch.isneginf(gl[1]).all()


@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_attention_without_some_pages(types):
    """Keys on pages that are not there take no part, whatever the pool holds:
    inside a tile, a whole tile, the first and the last page, all."""
    dt, ct = types
    c = Cache([200, 200, 200, 48], 24, 2, 64, dt, ct)
    there = torch.ones((4, 200), dtype=torch.bool)
    for b, i, bad in ((0, 1, -1), (1, 0, c.k_pages.shape[0]), (1, 8, -5), (2, 3, 2 ** 31 - 1), (2, 4, -2 ** 31), (2, 5, -1),
                      (3, 0, -1), (3, 1, -1)):
        c.table[b, i] = bad
        there[b, 24 * i:24 * i + 24] = False
    q = torch.randn((4, 10, 64), generator=torch.Generator().manual_seed(2)).to(dt)
    out, lse, tol, tl = attention(q, c, there)
    kp, vp, table, scales = c.device()
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    check(got, out, tol + 1e-30, "out")
    check(gl, lse, tl + 1e-30, "lse")
    assert not got[3].any() and torch.isneginf(gl[3]).all()
    # lengths below zero and beyond the table
    n = torch.tensor([-7, 2 ** 31 - 1, 0, 48], dtype=torch.int32)
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, n.cuda(), **scales)
    assert not got[0].any() and torch.isneginf(gl[0]).all() and not got[2].any()


@pytest.mark.parametrize("B,Hkv,wide", [(65, 1, 40), (150, 2, 24), (512, 1, 20), (513, 1, 20), (300, 64, 20)])
@pytest.mark.parametrize("types", [(F16, F16), (BF16, I8)], ids=ids)
def test_many_sequences(types, B, Hkv, wide):
    """More sequences than a wave has lanes, split and not: every length from
    nothing to the table's end, one far longer than the others."""
    dt, ct = types
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 60, (B,), generator=g).tolist()
    lens[B // 2], lens[0], lens[-1] = 16 * wide, 0, 33
    c = Cache(lens, 16, Hkv, 8, dt, ct, wide=wide)
    q = torch.randn((B, Hkv, 8), generator=g).to(dt)
    out, lse, tol, tl = attention(q, c)
    kp, vp, table, scales = c.device()
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    check(got, out, tol + 1e-30, "out")
    check(gl, lse, tl + 1e-30, "lse")


def test_no_pages_at_all():
    q = torch.randn(2, 4, 64, device="cuda")
    for shape, wide in (((0, 16, 2, 64), 3), ((4, 16, 2, 64), 0)):
        pool = torch.zeros(shape, device="cuda")
        table = torch.zeros((2, wide), dtype=torch.int32, device="cuda")
        n = torch.tensor([16, 5], dtype=torch.int32, device="cuda")
        out, lse = pkg.seq_paged_attention_forward(q, pool, pool, table, n)
        assert not out.any() and torch.isneginf(lse).all()
        k, v = pkg.seq_cache_read(pool, pool, table, n, 7)
        assert not k.any() and not v.any()


@pytest.mark.parametrize("types", [(F16, F16), (BF16, I8), (F16, I8), (F16, E4M3), (F32, I8)], ids=ids)
def test_values_of_very_different_sizes(types):
    """8-bit scales from 2^-20 to 2^8 in one sequence, keys that change sizes
    too, and bf16 queries from 2^-100 to 2^60."""
    dt, ct = types
    lens = [900, 257]
    c = Cache(lens, 32, 2, 64, dt, ct)
    g = torch.Generator().manual_seed(6)
    f = torch.exp2(torch.randint(-12, 9, c.v.shape[:3], generator=g).double())
    if ct == dt:
        c.v = (c.v * f[..., None]).to(dt).double()
        c._fill(c.v_pages, c.v.to(dt))
    else:
        s = f.float()
        c.v, c.v_top = c.v_codes * s.double()[..., None], float(s.max())
        c._fill(c.v_scale, s)
    q = torch.randn((2, 6, 64), generator=g)
    scale = 0.125
    if dt == BF16:
        q, scale = q * 2.0 ** 60, 0.125 * 2.0 ** -60
    q = q.to(dt)
    out, lse, tol, tl = attention(q, c, scale=scale)
    kp, vp, table, scales = c.device()
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), scale=scale, **scales)
    check(got, out, tol + 1e-30, "out")
    check(gl, lse, tl + 1e-30, "lse")


@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_values_that_are_not_finite(types):
    """NaN in a key or value reaches its own sequence and head only."""
    dt, ct = types
    c = Cache([300, 300, 300], 16, 2, 64, dt, ct)
    q = torch.randn((3, 8, 64), generator=torch.Generator().manual_seed(2)).to(dt)
    kp, vp, table, scales = c.device()
    clean, cl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    at = lambda b, p: (int(c.table[b, p // 16]), p % 16)
    kbad, vbad = (kp, vp) if ct == dt else (scales["k_scale"], scales["v_scale"])
    kbad[at(0, 250) + (1,)] = float("nan")
    vbad[at(1, 17) + (0,)] = float("nan")
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    assert torch.isnan(got[0, 4:]).all() and torch.isnan(gl[0, 4:]).all()
    assert torch.isnan(got[1, :4]).all() and torch.equal(gl[1], cl[1])
    for b, h in ((0, slice(0, 4)), (1, slice(4, 8)), (2, slice(0, 8))):
        assert torch.equal(got[b, h], clean[b, h]) and torch.equal(gl[b, h], cl[b, h])
    kp, vp, table, scales = c.device()
    q[2, 3, 7], q[0, 0, 0] = float("nan"), float("inf")
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    for b, h in ((2, 3), (0, 0)):  # scores of both signs and infinite
        assert torch.isnan(got[b, h]).all() and torch.isnan(gl[b, h])
        got[b, h], gl[b, h] = clean[b, h], cl[b, h]
    assert torch.equal(got, clean) and torch.equal(gl, cl)


@pytest.mark.parametrize("D,G", [(64, 1), (64, 5), (64, 8), (32, 1), (32, 8)])
@pytest.mark.parametrize("types", PAIRS, ids=ids)
def test_short_heads_side_by_side(types, D, G):
    """Two heads that lie next to each other, also where one of them is not
    finite, in a split sequence, a short one, an empty one and many whole ones."""
    dt, ct = types
    for lens, wide in (([2100, 70, 0, 1], 2000), ([40, 300, 0, 7] * 140, 20)):
        say("side by side", types, D, G, len(lens))
        c = Cache(lens, 16, 4, D, dt, ct, wide=wide)
        q = torch.randn((len(lens), 4 * G, D), generator=torch.Generator().manual_seed(4)).to(dt)
        bias = torch.randn((4 * G, 81), generator=torch.Generator().manual_seed(5))
        out, lse, tol, tl = attention(q, c, bias=bias, cap=15.0)
        kp, vp, table, scales = c.device()

        def run():
            return pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), cap=15.0, bias=bias.cuda(), **scales)
        got, gl = run()
        check(got, out, tol + 1e-30, "out")
        check(gl, lse, tl + 1e-30, "lse")
        # head 1's keys and head 2's values of a token of sequences 0 and 1
        if ct == I8:
            kbad, vbad = scales["k_scale"], scales["v_scale"]
        else:
            kbad, vbad = kp, vp
        for b, pos in ((0, 33), (1, 69 if len(lens) == 4 else 290)):
            at = (int(c.table[b, pos // 16]), pos % 16)
            nan = torch.full((1,), float("nan"), device="cuda").to(kbad.dtype)
            kbad[at + (1,)] = nan.expand(kbad[at + (1,)].shape) if kbad.dim() == 4 else nan[0]
            vbad[at + (2,)] = nan.expand(vbad[at + (2,)].shape) if vbad.dim() == 4 else nan[0]
        bad, bl = run()
        for b in range(2):
            if lens[b] > (33, 69 if len(lens) == 4 else 290)[b]:
                assert torch.isnan(bad[b, G:3 * G]).all() and torch.isnan(bl[b, G:2 * G]).all()
                assert torch.equal(bl[b, 2 * G:3 * G], gl[b, 2 * G:3 * G])
                bad[b, G:3 * G], bl[b, G:2 * G] = got[b, G:3 * G], gl[b, G:2 * G]
        assert torch.equal(bad, got) and torch.equal(bl, gl)


@pytest.mark.parametrize("types,Hkv", [((BF16, BF16), 16), ((F16, I8), 32), ((F32, F32), 8)], ids=["bf16", "f16-i8", "f32"])
def test_sequences_that_end_within_their_shares(types, Hkv):
    """Lengths that make a half more parts than the first estimate."""
    dt, ct = types
    c = Cache([800] * 25 + [799], 64, Hkv, 64, dt, ct)
    q = torch.randn((26, Hkv, 64), generator=torch.Generator().manual_seed(6)).to(dt)
    out, lse, tol, tl = attention(q, c)
    kp, vp, table, scales = c.device()
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    check(got, out, tol + 1e-30, "out")
    check(gl, lse, tl + 1e-30, "lse")


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F16, I8), (F16, E4M3)], ids=ids)
def test_strides_of_queries_results_tables_and_pages(types):
    dt, ct = types
    c = Cache([70, 33, 200], 16, 2, 64, dt, ct)
    q = torch.randn((3, 8, 64), generator=torch.Generator().manual_seed(2)).to(dt)
    kp, vp, table, scales = c.device()
    want, wl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales)
    packed = torch.full((3, 12, 72), float("nan"), dtype=dt, device="cuda")
    packed[:, 2:10, :64] = q.cuda()
    wide = torch.full((3, table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + table.shape[1]] = table
    raw = (lambda t: t.view(torch.uint8)) if ct == E4M3 else (lambda t: t)
    both = torch.zeros((kp.shape[0], 2, 16, 2, 72), dtype=raw(kp).dtype, device="cuda")  # keys and values in one page
    both[:, 0, :, :, :64], both[:, 1, :, :, :64] = raw(kp), raw(vp)
    both = both.view(ct)
    sc = {}
    if scales:
        s = torch.zeros((2, 2, kp.shape[0], 16), device="cuda")
        s[0], s[1] = scales["k_scale"].permute(2, 0, 1), scales["v_scale"].permute(2, 0, 1)
        sc = {"k_scale": s[0].permute(1, 2, 0), "v_scale": s[1].permute(1, 2, 0)}
    out = torch.full((8, 3, 64), float("nan"), dtype=dt, device="cuda").transpose(0, 1)
    got, gl = pkg.seq_paged_attention_forward(packed[:, 2:10, :64], both[:, 0, :, :, :64], both[:, 1, :, :, :64],
                                              wide[:, 2:2 + table.shape[1]], c.len.cuda(), out=out, **sc)
    assert got is out and torch.equal(got, want) and torch.equal(gl, wl)
    k, v = pkg.seq_cache_read(both[:, 0, :, :, :64], both[:, 1, :, :, :64], wide[:, 2:2 + table.shape[1]], c.len.cuda(), 200,
                              dtype=dt, **sc)
    k2, v2 = pkg.seq_cache_read(kp, vp, table, c.len.cuda(), 200, dtype=dt, **scales)
    assert torch.equal(k, k2) and torch.equal(v, v2)


@pytest.mark.parametrize("ct", [F16, I8], ids=["f16", "i8"])
def test_pages_beyond_4_gib(ct):
    """Offsets that pass 32 bits: three pages 2.4 GB apart."""
    c = Cache([40], 16, 1, 64, F16, ct, spare=0)
    size = c.k_pages.element_size()
    step = 1200000000 // size * 2
    big = torch.zeros(2 * step + 2 * 16 * 64, dtype=ct, device="cuda")
    at = lambda o: big[o:].as_strided((3, 16, 1, 64), (step, 64, 64, 1))
    kp, vp = at(0), at(16 * 64)
    scales = {}
    if c.k_scale is not None:
        scales = {"k_scale": c.k_scale.cuda(), "v_scale": c.v_scale.cuda()}
    q = torch.randn((1, 4, 64), generator=torch.Generator().manual_seed(2)).to(F16)
    out, lse, tol, tl = attention(q, c)
    kp.copy_(c.k_pages), vp.copy_(c.v_pages)
    got, gl = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, c.table.cuda(), c.len.cuda(), **scales)
    check(got, out, tol, "out")
    k, v = pkg.seq_cache_read(kp, vp, c.table.cuda(), c.len.cuda(), 40, dtype=F16, **scales)
    check(v, c.v, (U[F16] + 2.0 ** -23) * c.v.abs() + TINY[F16] + 1e-30, "read")
    kp.zero_(), vp.zero_()
    pkg.seq_cache_write(k, v, kp, vp, c.table.cuda(), **scales)
    k2, v2 = pkg.seq_cache_read(kp, vp, c.table.cuda(), c.len.cuda(), 40, dtype=F16, **scales)
    if ct == F16:
        assert torch.equal(k2, k) and torch.equal(v2, v)
    else:  # rounded once more: by at most half a step of the head's largest / 127, and fp16's own
        top = v.float().abs().amax(-1, keepdim=True)
        assert ((v2.float() - v.float()).abs() <= top * (0.5 / 127 * (1 + 2.0 ** -20) + 2.0 ** -11)).all()


def status(fn, *a, **k):
    with pytest.raises(pkg.Im2winError) as e:
        fn(*a, **k)
    return e.value.status


def test_refusals_with_buffers():
    EALIGN, EWORKSPACE, EOVERLAP, EBUFFER = -2, -6, -7, -8
    pool, other = torch.zeros(8, 16, 2, 64, device="cuda"), torch.zeros(8, 16, 2, 64, device="cuda")
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    k = torch.zeros(2, 5, 2, 64, device="cuda")
    w, r, a = pkg.seq_cache_write, pkg.seq_cache_read, pkg.seq_paged_attention_forward
    assert status(w, k, k, pool, pool, table) == EOVERLAP
    assert status(w, pool[:2, :5], k, pool, other, table) == EOVERLAP
    assert status(w, k, k, pool[:1].expand(8, 16, 2, 64), other, table) == EOVERLAP
    ints = pool.view(torch.int32).view(-1)
    assert status(w, k, k, pool, other, ints[:8].view(2, 4)) == EOVERLAP
    assert status(w, k, k, pool, other, table, ints[8:10]) == EOVERLAP
    assert status(w, k, k, pool, other, table, n, ints[8:10]) == EOVERLAP
    codes = torch.zeros(8, 16, 2, 64, dtype=torch.int8, device="cuda")
    more, scale = codes.clone(), torch.zeros(8, 16, 2, device="cuda")
    assert status(w, k, k, codes, more, table, k_scale=scale, v_scale=scale) == EOVERLAP
    assert status(w, k, k, codes, more, table, k_scale=codes.view(torch.float32).view(-1)[:256].view(8, 16, 2), v_scale=scale) == EOVERLAP
    assert status(r, pool, other, table, n, 5, k=k, v=k) == EOVERLAP
    assert status(r, pool, other, table, n, 5, k=k, v=pool[:2, :5]) == EOVERLAP
    q = torch.zeros(2, 4, 64, device="cuda")
    assert status(a, q, pool, pool, table, n, out=q) == EOVERLAP
    assert status(a, q, pool, pool, table, n, out=pool[:1, :2].view(1, 4, 64).expand(2, 4, 64)) == EOVERLAP
    assert status(a, torch.zeros(2, 4, 66, device="cuda")[..., :64], pool, pool, table, n) == EALIGN
    long = torch.zeros(2, 400, dtype=torch.int32, device="cuda")
    need = pkg.seq_paged_attention_workspace_bytes(q, pool, pool, long)
    assert need > 0
    assert status(a, q, pool, pool, long, n, ws=torch.zeros(need - 16, dtype=torch.uint8, device="cuda")) == EWORKSPACE
    host = torch.zeros(8, 16, 2, 64)
    assert status(w, k.cpu(), k.cpu(), host, host.clone(), table.cpu()) == EBUFFER
    assert status(r, host, host, table.cpu(), n.cpu(), 5) == EBUFFER
    assert status(a, q.cpu(), host, host, table.cpu(), n.cpu()) == EBUFFER


def test_same_bits_every_time():
    c = Cache([3000, 777], 64, 2, 128, BF16, I8)
    q = torch.randn((2, 32, 128), generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    kp, vp, table, scales = c.device()
    n = c.len.cuda()
    first = pkg.seq_paged_attention_forward(q, kp, vp, table, n, **scales)
    for _ in range(4):
        again = pkg.seq_paged_attention_forward(q, kp, vp, table, n, **scales)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


@pytest.mark.parametrize("types", [(BF16, BF16), (F16, I8)], ids=ids)
def test_graphs_and_streams(types):
    """A serving step captured (turn, write, attend) and replayed as the
    sequences grow, two graphs on one workspace among them, and the same calls
    on another stream."""
    dt, ct = types
    c = Cache([60, 15, 130], 16, 2, 64, dt, ct, wide=200)
    kp, vp, table, scales = c.device()
    spare = kp.shape[0]
    grow = lambda t: torch.cat([t.view(torch.int8) if t.dtype == E4M3 else t, torch.zeros((9, *t.shape[1:]), dtype=t.dtype, device="cuda")])
    kp, vp, scales = grow(kp), grow(vp), {k: grow(s) for k, s in scales.items()}
    for b, n in enumerate(c.lens):  # room for three more pages each
        used = (n + 15) // 16
        table[b, used:used + 3] = torch.arange(spare + 3 * b, spare + 3 * b + 3)
    n = c.len.cuda()
    freq = pkg.seq_rotary_frequencies(64)
    x = torch.randn((3, 1, 8 + 4, 64), generator=torch.Generator().manual_seed(3)).to(dt).cuda()
    ws = torch.empty(max(16, pkg.seq_paged_attention_workspace_bytes(x[:, 0, :8], kp, vp, table, **scales)), dtype=torch.uint8, device="cuda")

    def step(kp, vp, scales, n, ws=None, stream=None):
        y = pkg.seq_rotary_forward(x[:, :, :10], freq, n, stream=stream)
        pkg.seq_cache_write(y[:, :, 8:], x[:, :, 10:], kp, vp, table, n, stream=stream, **scales)
        if stream is None:
            return pkg.seq_paged_attention_forward(y[:, 0, :8], kp, vp, table, n + 1, ws=ws, **scales)
        with torch.cuda.stream(stream):
            m = n + 1
        return pkg.seq_paged_attention_forward(y[:, 0, :8], kp, vp, table, m, stream=stream, **scales)
    step(kp.clone(), vp.clone(), {k: s.clone() for k, s in scales.items()}, n)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step(kp, vp, scales, n, ws))
    side = torch.cuda.Stream()
    for k in range(6):
        x.copy_(torch.randn((3, 1, 12, 64), generator=torch.Generator().manual_seed(30 + k)).to(dt))
        mine = [kp.clone(), vp.clone(), {a: s.clone() for a, s in scales.items()}]
        torch.cuda.synchronize()
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        want, wl = step(*mine, n)
        out, lse = outs[k % 2]
        assert torch.equal(out, want) and torch.equal(lse, wl), k
        same(kp, mine[0], "keys")
        same(vp, mine[1], "values")
        side.wait_stream(torch.cuda.current_stream())
        got, gl = step(*mine, n, stream=side)
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(gl, wl), k
        n += 1


@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_the_operators_together(dt):
    """A block's serving path against attention over whole sequences: prompts
    in pieces (turn, write, read back, attend), then tokens one by one (turn,
    write, attend over the pages)."""
    B, H, Hkv, D, page, L = 3, 6, 2, 64, 16, 75
    g = torch.Generator().manual_seed(8)
    qkv = torch.randn((B, L, H + 2 * Hkv, D), generator=g).to(dt).cuda()
    freq = pkg.seq_rotary_frequencies(48, factor=2.0, trained=32)
    turned = pkg.seq_rotary_forward(qkv[:, :, :H + Hkv], freq)
    want, _ = pkg.seq_attention_forward(turned[:, :, :H], turned[:, :, H:], qkv[:, :, H + Hkv:], causal=True)
    kp, vp = (torch.full((B * 5, page, Hkv, D), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    table = torch.randperm(B * 5, generator=g).int().view(B, 5).cuda()
    n = torch.zeros(B, dtype=torch.int32, device="cuda")
    outs = []
    for m in (20, 27, 14) + (1,) * (L - 61):
        at = int(n[0])
        part = qkv[:, at:at + m]
        y = pkg.seq_rotary_forward(part[:, :, :H + Hkv], freq, n)
        pkg.seq_cache_write(y[:, :, H:], part[:, :, H + Hkv:], kp, vp, table, n)
        n += m
        if m > 1:
            k, v = pkg.seq_cache_read(kp, vp, table, n, at + m)
            outs.append(pkg.seq_attention_forward(y[:, :, :H], k, v, causal=True, align_end=True, kv_len=n)[0])
        else:
            outs.append(pkg.seq_paged_attention_forward(y[:, 0, :H], kp, vp, table, n)[0][:, None])
    got = torch.cat(outs, 1)
    # both round P and the result (u each) and sum in fp32; |out| <= max |v|
    u = U[dt]
    size = float(qkv[:, :, H + Hkv:].abs().max())
    assert float((got.double() - want.double()).abs().max()) <= (4 * u + 2.0 ** -18) * size
