"""Attention over 8-bit pages whose numbers come near the ends of the type's range."""
import pytest
import torch

import paper_2608_20725_amd as pkg
from gpu_util import say
from seq_cache_ref import E4M3, Cache, attention
from seq_ref import check

pytestmark = pytest.mark.gpu

F32, F16, BF16, I8 = torch.float32, torch.float16, torch.bfloat16, torch.int8
NAMES = {F32: "f32", F16: "f16", BF16: "bf16", I8: "i8", E4M3: "e4m3"}
WIDE_OVER_CODES = [(F32, I8), (BF16, I8), (F32, E4M3), (BF16, E4M3)]
ids = lambda v: "-".join(NAMES[t] for t in v) if isinstance(v[0], torch.dtype) else None


def scaled(c, name, factor):
    """The cache's keys or values times ``factor`` [B][longest][Hkv] or a number, by their scales."""
    s = getattr(c, name + "_codes")
    old = getattr(c, name).abs().amax(-1) / s.abs().amax(-1).clamp(min=1)
    new = (old * factor).float()
    setattr(c, name, s * new.double()[..., None])
    setattr(c, name + "_top", float(new.max()))
    c._fill(getattr(c, name + "_scale"), new)


def attend(q, c, **opts):
    kp, vp, table, scales = c.device()
    need = pkg.seq_paged_attention_workspace_bytes(q.cuda(), kp, vp, table, **scales)
    out, lse = pkg.seq_paged_attention_forward(q.cuda(), kp, vp, table, c.len.cuda(), **scales, **opts)
    return out, lse, need > 0


# Lengths, table, key/value heads, queries each, channels; whether the keys are split.
SHAPES = [([1], None, 1, 1, 64, False), ([1, 700, 0, 5000], None, 2, 4, 64, True), ([3000], 2000, 1, 5, 128, True),
          ([40, 300, 1] * 50, 20, 2, 2, 128, False), ([900, 33], 500, 2, 17, 72, True), ([2500, 3], None, 1, 40, 64, True),
          ([300, 12], 20, 3, 3, 32, False)]


@pytest.mark.parametrize("e", [108, 112, 116, 120, 123])
@pytest.mark.parametrize("types", WIDE_OVER_CODES, ids=ids)
def test_values_near_the_largest_number(types, e):
    """Every result is a mean of values, so it is within the type's range where they are (up to 2^(e + 3.2))."""
    dt, ct = types
    for k, (lens, wide, Hkv, G, D, split) in enumerate(SHAPES):
        say("large values", types, e, k)
        c = Cache(lens, 16, Hkv, D, dt, ct, wide=wide, seed=k)
        scaled(c, "v", 2.0 ** e)
        q = (torch.randn((len(lens), Hkv * G, D), generator=torch.Generator().manual_seed(k)) * 2.0 ** -4).to(dt)
        out, lse, tol, tl = attention(q, c)
        assert torch.isfinite(out).all() and float(out.abs().max()) < 2.0 ** 127
        got, gl, parts = attend(q, c)
        assert parts == split
        check(got, out, tol + 1e-30, "out %d" % k)
        check(gl, lse, tl + 1e-30, "lse %d" % k)


@pytest.mark.parametrize("r", [30, 45, 100, 200])
@pytest.mark.parametrize("types", WIDE_OVER_CODES + [(F16, I8), (F16, E4M3)], ids=ids)
def test_large_values_that_are_not_looked_at(types, r):
    """A token whose weight is nothing, with a value 2^r times the others', takes no bit of theirs: in its tile, in
    one before and in one behind, in its part of split keys and in whole sequences."""
    dt, ct = types
    least = -90 if r == 200 and dt != F16 else 0  # the others' size
    r = min(r, 110) if dt == F16 else r
    for k, (lens, wide, at) in enumerate((([2], None, 0), ([700, 300], None, 0), ([700, 300], None, 299), ([260] * 40, 20, 130),
                                          ([6000, 3000], 500, 2900))):
        say("not looked at", types, r, k)
        D = 64 if k % 2 else 128
        c = Cache(lens, 16, 2, D, dt, ct, wide=wide, seed=k)
        f = torch.full(c.v.shape[:3], 2.0 ** least, dtype=torch.float64)
        f[:, at] *= 2.0 ** r
        scaled(c, "v", f)
        q = torch.randn((len(lens), 4, D), generator=torch.Generator().manual_seed(k)).to(dt)
        # the bias of its distance puts its score 400 below the others'
        n, R = min(lens), 1000
        c.len = torch.full_like(c.len, n)
        bias = torch.zeros(4, 2 * R + 1)
        bias[:, R - (n - 1 - at)] = -400.0
        _, lse, _, tl = attention(q, c, bias=bias)
        # and the bound is that of the others
        there = torch.ones(c.v.shape[:2], dtype=torch.bool)
        there[:, at] = False
        c.v_codes[:, at], c.v[:, at] = 0, 0
        c.v_top *= 2.0 ** -r
        near, _, tol, _ = attention(q, c, there, bias=bias)
        got, gl, _ = attend(q, c, bias=bias.cuda())
        check(got, near, tol + 1e-40, "out %d" % k)
        check(gl, lse, tl + 1e-30, "lse %d" % k)


@pytest.mark.parametrize("e,size", [(-110, 0.5), (-60, 0.5), (60, 0.5), (100, 0.5), (118, 64.0)])
@pytest.mark.parametrize("types", WIDE_OVER_CODES, ids=ids)
def test_large_queries_of_small_keys(types, e, size):
    """Queries of 2^e over keys of 2^-e, all of one sign: ordinary scores."""
    dt, ct = types
    for k, (lens, wide, Hkv, G, D, split) in enumerate(SHAPES):
        say("large queries", types, e, k)
        c = Cache(lens, 16, Hkv, D, dt, ct, wide=wide, seed=k)
        c.k, c.k_codes = c.k.abs(), c.k_codes.abs()
        c._fill(c.k_pages, c.k_codes.to(ct))
        scaled(c, "k", 2.0 ** -e)
        q = (torch.randn((len(lens), Hkv * G, D), generator=torch.Generator().manual_seed(k)).abs() * 2.0 ** e).to(dt)
        out, lse, tol, tl = attention(q, c, scale=size / D)
        got, gl, _ = attend(q, c, scale=size / D)
        check(got, out, tol + 1e-30, "out %d" % k)
        check(gl, lse, tl + 1e-30, "lse %d" % k)


@pytest.mark.parametrize("B", [1, 7])
@pytest.mark.parametrize("ct", [F16, I8], ids=["f16", "i8"])
def test_as_many_heads_as_are_taken(ct, B):
    """Parts rounded up to the XCDs would pass 2^32 lanes here: 2^21 heads a sequence, the most with B*H < 2^24."""
    H, g = 1 << 21, torch.Generator("cuda").manual_seed(B)
    codes = lambda: torch.randint(-127, 128, (B, 1, H, 8), generator=g, device="cuda", dtype=torch.int8)
    k, v = codes(), codes()
    scales = {}
    if ct == F16:
        k, v = k.to(F16) / 64, v.to(F16) / 64
    else:
        scales = {"k_scale": torch.full((B, 1, H), 2.0 ** -6, device="cuda"), "v_scale": torch.full((B, 1, H), 2.0 ** -6, device="cuda")}
    q = torch.randint(-8, 9, (B, H, 8), generator=g, device="cuda").to(F16)
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None]
    n = torch.ones(B, dtype=torch.int32, device="cuda")
    out, lse = pkg.seq_paged_attention_forward(q, k, v, table, n, scale=0.25, **scales)
    values = lambda t: (t.float() * (2.0 ** -6 if ct == I8 else 1.0))[:, 0]
    # one key: its value, and its score (multiples of 2^-8 below 2^9, exact in fp32) times log2(e), plus and less 14 of
    # the weights' 2^14, and times ln(2): four roundings of values up to |1.45 score| + 14
    assert torch.equal(out, values(v).to(F16))
    score = (q.float() * values(k)).sum(-1) * 0.25
    assert ((lse - score).abs() <= 2.0 ** -21 * (2 * score.abs() + 14)).all()
