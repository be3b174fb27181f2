"""Attention forward and backward against the plain form in 64 bits: types,
head layouts, lengths, masks, strides, what masked places hold, repeated
calls, streams and graphs."""
import math

import pytest
import torch

import paper_2608_20725_amd as pkg
from seq_ref import Attention, check

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
DTYPES = [F32, F16, BF16]
ids = lambda v: str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None


def draw(B, Lq, Lk, H, Hk, D, dtype, seed=0, R=0):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g).to(dtype)
    x = {"q": t(B, Lq, H, D), "k": t(B, Lk, Hk, D), "v": t(B, Lk, Hk, D), "dout": t(B, Lq, H, D)}
    bias = torch.randn((H, 2 * R + 1), generator=g) if R else None
    return x, bias


def to_gpu(v):
    return v.cuda() if isinstance(v, torch.Tensor) else v


def run(x, bias, opts, backward=True, check_values=True):
    o = {k: to_gpu(v) for k, v in opts.items()}
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    out, lse = pkg.seq_attention_forward(q, k, v, bias=to_gpu(bias), **o)
    ref = Attention(x["q"], x["k"], x["v"], bias=bias, **opts)
    if check_values:
        to, tl = ref.tolerances()
        check(out, ref.out.transpose(1, 2), to + 1e-30, "out")
        check(lse, ref.lse, tl + 1e-30, "lse")
    if not backward:
        return out, lse
    grads = pkg.seq_attention_backward(do, q, k, v, out, lse, bias=to_gpu(bias), **o)
    want, tol = ref.grads(x["dout"], out.cpu(), lse.cpu())
    for name, a, w, t in zip(("dq", "dk", "dv", "dstrip"), grads, want, tol):
        if w is None:
            assert a is None
        else:
            check(a, w, t, name)
    return (out, lse) + tuple(grads)


SHAPES = [
    # B, Lq, Lk, H, Hk, D
    (1, 1, 1, 1, 1, 8),
    (2, 1, 70, 4, 2, 64),
    (1, 33, 1, 2, 2, 32),
    (2, 65, 65, 2, 1, 40),
    (1, 127, 200, 3, 3, 96),
    (1, 130, 64, 4, 1, 128),
    (2, 257, 129, 2, 2, 72),
    (1, 31, 300, 6, 2, 104),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_plain(shape, dtype):
    x, _ = draw(*shape, dtype)
    run(x, None, {})


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bias_cap_causal(shape, dtype):
    for R, causal, end, cap in ((1, False, False, 0.0), (17, True, True, 5.0), (200, True, False, 30.0),
                                (40, False, True, 0.0)):
        x, bias = draw(*shape, dtype, seed=R, R=R)
        run(x, bias, {"causal": causal, "align_end": end, "cap": cap})


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_and_prefix(dtype, causal):
    B, L = 5, 150
    x, bias = draw(B, L, L, 4, 2, 64, dtype, R=30)
    lens = torch.tensor([150, 0, 1, 64, 97], dtype=torch.int32)
    run(x, bias, {"causal": causal, "kv_len": lens})
    run(x, None, {"causal": causal, "kv_len": lens, "align_end": True})
    if causal:
        pre = torch.tensor([10, 5, 0, 150, 65], dtype=torch.int32)
        run(x, bias, {"causal": True, "kv_len": lens, "prefix": pre})
        run(x, None, {"causal": True, "prefix": pre})
        # values outside 0 .. Lk are taken as the nearest
        run(x, None, {"causal": True, "kv_len": torch.tensor([151, -3, 1000000, 64, 97], dtype=torch.int32)})


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_documents(dtype):
    B, L = 3, 333
    g = torch.Generator().manual_seed(5)
    rows = [torch.tensor([0] * 64 + [1] * 64 + [2] * 5 + [7] * 150 + [-1] * 50),
            torch.randint(-1, 4, (L,), generator=g),                      # any order
            torch.full((L,), -1)]                                          # no query sees anything
    doc = torch.stack(rows).to(torch.int32)
    x, bias = draw(B, L, L, 4, 2, 64, dtype, R=20)
    run(x, bias, {"q_doc": doc, "k_doc": doc})
    out = run(x, None, {"q_doc": doc, "k_doc": doc, "causal": True, "cap": 20.0})
    assert (out[0][2] == 0).all() and torch.isinf(out[1][2]).all()
    for t in out[2:5]:
        assert (t[2] == 0).all()
    # other documents on the key side, lengths that cut them
    kd = torch.stack([rows[1][torch.randperm(L, generator=g)]] * 3).to(torch.int32)
    run(x, None, {"q_doc": doc, "k_doc": kd, "kv_len": torch.tensor([333, 100, 200], dtype=torch.int32)})


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("hold", [math.nan, math.inf, -math.inf, "largest"], ids=str)
def test_masked_places_hold_anything(dtype, hold):
    """Keys, values, queries and gradients that no pair uses do not reach any
    result: the same bits as with zeros there."""
    hold = torch.finfo(dtype).max if hold == "largest" else hold
    L = 200
    x, bias = draw(3, L, L, 2, 1, 64, dtype, R=10)
    doc = torch.zeros((3, L), dtype=torch.int32)
    doc[:, 70:90] = -1
    doc[1, 90:] = 1
    lens = torch.tensor([200, 200, 130], dtype=torch.int32)
    opts = {"q_doc": doc, "k_doc": doc, "kv_len": lens, "causal": True}
    gone = doc < 0
    gone_k = gone | (torch.arange(L)[None] >= lens[:, None])
    res = []
    for value in (0.0, hold):
        y = {n: t.clone() for n, t in x.items()}
        for n in ("q", "dout"):
            y[n][gone] = value
        for n in ("k", "v"):
            y[n][gone_k] = value
        o = {k: to_gpu(v) for k, v in opts.items()}
        q, k, v, do = (y[n].cuda() for n in ("q", "k", "v", "dout"))
        out, lse = pkg.seq_attention_forward(q, k, v, bias=bias.cuda(), **o)
        res.append((out, lse) + pkg.seq_attention_backward(do, q, k, v, out, lse, bias=bias.cuda(), **o))
    for a, b in zip(*res):
        assert not torch.isnan(b).any()
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_values_not_finite_reach_only_their_pairs(dtype):
    """A value (key, ..) that is not finite makes NaN or infinity of exactly
    the results it takes part in, also within one tile."""
    L = 96
    x, _ = draw(1, L, L, 2, 2, 64, dtype)
    doc = torch.zeros((1, L), dtype=torch.int32)
    doc[:, 40:] = 1
    x["v"][0, 20, 1, 3] = math.nan
    x["v"][0, 50, 0, 7] = math.inf
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    out, lse = pkg.seq_attention_forward(q, k, v, causal=True, q_doc=doc.cuda(), k_doc=doc.cuda())
    bad = ~torch.isfinite(out.cpu())
    want = torch.zeros_like(bad)
    want[0, 20:40, 1, 3] = True
    want[0, 50:, 0, 7] = True
    assert torch.equal(bad, want)
    assert torch.isfinite(lse).all()
    # backward: a dout row
    x, _ = draw(1, L, L, 1, 1, 64, dtype)
    x["dout"][0, 20, 0, 3] = math.nan
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    out, lse = pkg.seq_attention_forward(q, k, v, causal=True, q_doc=doc.cuda(), k_doc=doc.cuda())
    dq, dk, dv, _ = pkg.seq_attention_backward(do, q, k, v, out, lse, causal=True, q_doc=doc.cuda(), k_doc=doc.cuda())
    assert torch.isnan(dq[0, 20]).all() and torch.isnan(dk[0, :21]).any(-1).all() and torch.isnan(dv[0, :21, :, 3]).all()
    rest = torch.ones(L, dtype=torch.bool)
    rest[20] = False
    assert torch.isfinite(dq.cpu()[0, rest]).all()
    assert torch.isfinite(dk[0, 21:]).all() and torch.isfinite(dv[0, 21:]).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_strides(dtype):
    """q, k, v and their gradients as columns of one packed tensor, heads
    before tokens, broadcast keys."""
    B, L, H, D = 2, 90, 3, 64
    x, bias = draw(B, L, L, H, H, D, dtype, R=7)
    want = run(x, bias, {"causal": True})
    packed = torch.stack([x["q"], x["k"], x["v"]], 2).cuda()
    q, k, v = packed.unbind(2)
    grads = torch.full_like(packed, 7)
    wide = torch.full((B, L, H, 2 * D), 7, dtype=dtype, device="cuda")
    out, lse = pkg.seq_attention_forward(q, k, v, bias=bias.cuda(), causal=True, out=wide[..., D:])
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and (wide[..., :D] == 7).all()
    dq, dk, dv = grads.unbind(2)
    do = x["dout"].transpose(1, 2).contiguous().transpose(1, 2).cuda()   # heads before tokens in memory
    got = pkg.seq_attention_backward(do, q, k, v, out, lse, bias=bias.cuda(), causal=True, dq=dq, dk=dk, dv=dv)
    for a, b in zip(got, want[2:]):
        assert torch.equal(a, b)
    # one key and value sequence for the whole batch
    k1, v1 = x["k"][:1].expand(B, L, H, D), x["v"][:1].expand(B, L, H, D)
    ref = pkg.seq_attention_forward(x["q"].cuda(), k1.contiguous().cuda(), v1.contiguous().cuda())
    got = pkg.seq_attention_forward(x["q"].cuda(), x["k"][:1].cuda().expand(B, L, H, D),
                                    x["v"][:1].cuda().expand(B, L, H, D))
    assert torch.equal(ref[0], got[0])


def test_offsets_beyond_32_bits():
    """A cache whose token stride puts late keys more than 4 GiB from the first."""
    L, D, stride = 600, 64, 1 << 22                        # elements: 8 MiB a token
    big = torch.empty(L * stride, dtype=F16, device="cuda")
    x, _ = draw(1, 40, L, 1, 1, D, F16)
    k = big.as_strided((1, L, 1, D), (L * stride, stride, D, 1))
    v = big[D:].as_strided((1, L, 1, D), (L * stride, stride, D, 1))
    k.copy_(x["k"])
    v.copy_(x["v"])
    q, do = x["q"].cuda(), x["dout"].cuda()
    out, lse = pkg.seq_attention_forward(q, k, v, causal=True, align_end=True)
    ref = pkg.seq_attention_forward(q, x["k"].cuda(), x["v"].cuda(), causal=True, align_end=True)
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
    a = pkg.seq_attention_backward(do, q, k, v, out, lse, causal=True, align_end=True)
    b = pkg.seq_attention_backward(do, q, x["k"].cuda(), x["v"].cuda(), out, lse, causal=True, align_end=True)
    for s, t in zip(a[:3], b[:3]):
        assert torch.equal(s, t)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_nothing_to_do(dtype):
    z = lambda *s: torch.zeros(s, dtype=dtype, device="cuda")
    for B, Lq, Lk in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        q, k, v = z(B, Lq, 2, 32), z(B, Lk, 2, 32) + 1, z(B, Lk, 2, 32) + 1
        bias = torch.zeros((2, 5), device="cuda")
        out, lse = pkg.seq_attention_forward(q, k, v, bias=bias, causal=True)
        assert (out == 0).all() and (lse == -math.inf).all()
        dq, dk, dv, ds = pkg.seq_attention_backward(q, q, k, v, out, lse, bias=bias, causal=True)
        for t in (dq, dk, dv, ds):
            assert (t == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_large_scores(dtype):
    """Scores of hundreds, and an f16 gradient of a loss scaled by 2^12."""
    x, bias = draw(1, 100, 100, 2, 2, 64, dtype, R=3)
    x["q"] = x["q"] * 16
    run(x, bias * 30, {"causal": True})
    x, _ = draw(1, 100, 100, 2, 2, 64, dtype)
    x["dout"] = x["dout"] * 4096
    run(x, None, {})
    x["dout"] = (x["dout"].float() * 2.0 ** -24).to(dtype)
    run(x, None, {})


@pytest.mark.parametrize("dtype", [F32])
def test_gradient_against_differences(dtype):
    """Directional derivatives of sum(out*dout) in q, k, v and the strip.

    Central differences with step h: truncation h^2/6 times the third
    derivative (of order 1 to 10 times the first here), rounding 2^-23 of the
    sum's terms (2*70*2*32 terms of size 1: below 0.01) over h."""
    B, L, H, D, h = 2, 70, 2, 32, 2.0 ** -6
    x, bias = draw(B, L, L, H, H, D, dtype, R=9)
    opts = {"causal": True, "cap": 3.0}
    t = {n: v.cuda() for n, v in x.items()}
    t["bias"] = bias.cuda()
    out, lse = pkg.seq_attention_forward(t["q"], t["k"], t["v"], bias=t["bias"], **opts)
    grads = pkg.seq_attention_backward(t["dout"], t["q"], t["k"], t["v"], out, lse, bias=t["bias"], **opts)
    g = torch.Generator().manual_seed(9)
    for name, grad in zip(("q", "k", "v", "bias"), grads):
        way = torch.randn(t[name].shape, generator=g).cuda()
        way = way / way.norm()
        vals = []
        for s in (h, -h):
            y = dict(t)
            y[name] = t[name] + s * way
            o, _ = pkg.seq_attention_forward(y["q"], y["k"], y["v"], bias=y["bias"], **opts)
            vals.append(float((o.double() * t["dout"].double()).sum()))
        diff = (vals[0] - vals[1]) / (2 * h)
        want = float((grad.double() * way.double()).sum())
        size = float(grad.double().norm())
        assert abs(diff - want) <= 2e-3 * size, (name, diff, want, size)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_same_bits_again_and_on_another_stream(dtype):
    x, bias = draw(2, 500, 500, 4, 2, 64, dtype, R=100)
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    bias = bias.cuda()

    def both(**kw):
        out, lse = pkg.seq_attention_forward(q, k, v, bias=bias, causal=True, **kw)
        return (out, lse) + pkg.seq_attention_backward(do, q, k, v, out, lse, bias=bias, causal=True, **kw)
    first = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for kw in ({}, {"stream": side}, {"stream": side.cuda_stream}):
        again = both(**kw)
        torch.cuda.synchronize()
        for a, b in zip(first, again):
            assert torch.equal(a, b)


def test_graph():
    x, bias = draw(1, 300, 300, 2, 2, 64, BF16, R=20)
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    bias = bias.cuda()

    def both():
        out, lse = pkg.seq_attention_forward(q, k, v, bias=bias, causal=True)
        return (out, lse) + pkg.seq_attention_backward(do, q, k, v, out, lse, bias=bias, causal=True)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for r in range(3):
        q.copy_(torch.randn_like(q))
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, held):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(1, 1, 5000, 8, 2, 64), (3, 1, 1025, 32, 1, 128), (2, 3, 700, 8, 1, 96), (2, 8, 333, 4, 1, 32),
                                   (70, 1, 300, 8, 8, 40), (1, 32, 2111, 1, 1, 128)], ids=str)
def test_few_rows_long_cache(shape, dtype):
    """Single tokens (and a few) over caches that several workgroups split."""
    B, Lq, Lk, H, Hk, D = shape
    x, bias = draw(*shape, dtype, seed=Lk, R=50)
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, Lk + 1, (B,), generator=g).to(torch.int32)
    lens[0] = Lk
    run(x, None, {}, backward=False)
    run(x, bias, {"causal": True, "align_end": True, "kv_len": lens, "cap": 20.0}, backward=False)
    doc = torch.randint(-1, 3, (B, Lk), generator=g).to(torch.int32)
    run(x, bias, {"align_end": True, "kv_len": lens, "q_doc": doc[:, -Lq:].contiguous(), "k_doc": doc}, backward=False)
    pre = torch.randint(0, Lk, (B,), generator=g).to(torch.int32)
    run(x, bias, {"causal": True, "prefix": pre}, backward=False)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_few_rows_masked_places(dtype):
    """What a cache holds beyond its length, and in other documents, does not
    reach the result."""
    B, Lk = 3, 900
    x, bias = draw(B, 2, Lk, 4, 2, 64, dtype, R=10)
    lens = torch.tensor([900, 0, 415], dtype=torch.int32)
    doc = torch.zeros((B, Lk), dtype=torch.int32)
    doc[:, 100:150] = 2
    o = {"kv_len": lens.cuda(), "k_doc": doc.cuda(), "q_doc": torch.zeros((B, 2), dtype=torch.int32, device="cuda")}
    gone = (doc != 0) | (torch.arange(Lk)[None] >= lens[:, None])
    res = []
    for value in (0.0, math.nan, math.inf):
        k, v = x["k"].clone(), x["v"].clone()
        k[gone] = value
        v[gone] = value
        res.append(pkg.seq_attention_forward(x["q"].cuda(), k.cuda(), v.cuda(), bias=bias.cuda(), **o))
    for other in res[1:]:
        for a, b in zip(res[0], other):
            assert not torch.isnan(b).any() and torch.equal(a, b)
    assert (res[0][0][1] == 0).all() and (res[0][1][1] == -math.inf).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_rows_do_not_depend_on_their_batch(dtype):
    """A sequence gives the same bits alone and among others (one chunking)."""
    x, _ = draw(9, 200, 200, 4, 2, 64, dtype)
    q, k, v = (x[n].cuda() for n in "qkv")
    whole = pkg.seq_attention_forward(q, k, v, causal=True)
    for b in (0, 4, 8):
        one = pkg.seq_attention_forward(q[b:b + 1], k[b:b + 1], v[b:b + 1], causal=True)
        assert torch.equal(one[0][0], whole[0][b]) and torch.equal(one[1][0], whole[1][b])


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("Lk", [1, 33, 95, 417])
def test_few_rows_documents_end_with_the_cache(dtype, Lk):
    """Ids are taken from the keys there are: what lies behind them in memory
    has no influence, be it the query's document."""
    x, _ = draw(2, 1, Lk, 4, 2, 64, dtype, seed=Lk)
    doc = torch.randint(0, 2, (2, Lk), generator=torch.Generator().manual_seed(Lk)).to(torch.int32)
    doc[:, 0] = 1
    q, k, v = (x[n].cuda() for n in "qkv")
    ones = torch.ones((2, 1), dtype=torch.int32, device="cuda")
    res = []
    for behind in (-1, 0, 1):
        room = torch.full((2 * Lk + 64,), behind, dtype=torch.int32, device="cuda")
        room[:2 * Lk] = doc.flatten().cuda()
        res.append(pkg.seq_attention_forward(q, k, v, q_doc=ones, k_doc=room[:2 * Lk].view(2, Lk)))
    run(x, None, {"q_doc": ones.cpu(), "k_doc": doc}, backward=False)
    for other in res[1:]:
        assert torch.equal(res[0][0], other[0]) and torch.equal(res[0][1], other[1])
