"""Sequence operators at the edges of their ranges: scores that are NaN, caps
far above the scores, what padding holds, empty calls of every kernel, odd
layouts, other streams, keys that several workgroups share."""
import math

import pytest
import torch

import paper_2608_20725_amd as pkg
from seq_ref import Attention, allowed, check
from test_gpu_seq_attention import BF16, DTYPES, F16, F32, draw, ids, run, to_gpu
from test_gpu_seq_norm import test_layer_norm as layer_norm_case

pytestmark = pytest.mark.gpu


def nan_rows(x, lens, **opts):
    """([B][H][Lq] rows with a NaN among their scores) by the definition."""
    B, Lq, H, D = x["q"].shape
    Lk, Hk = x["k"].shape[1:3]
    i, j = torch.arange(Lq)[:, None], torch.arange(Lk)[None, :]
    bad = torch.zeros((B, H, Lq), dtype=torch.bool)
    for b in range(B):
        n = int(lens[b])
        ok = (j < n) & (j <= i + (n - Lq if opts.get("align_end") else 0))
        for h in range(H):
            gone = torch.isnan(x["q"][b, :, h]).any(-1)[:, None] | torch.isnan(x["k"][b, :, h * Hk // H]).any(-1)[None, :]
            bad[b, h] = (ok & gone).any(1)
    return bad


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape,end", [((2, 70, 4, 2, 64), True), ((1, 900, 4, 1, 40), True), ((100, 100, 2, 2, 64), False),
                                       ((130, 1100, 4, 2, 96), False), ((200, 1100, 2, 1, 128), True)], ids=str)
def test_scores_that_are_nan(shape, end, dtype):
    """A query one of whose scores is NaN has out and lse NaN, also where all
    of them are: it is not taken for one without pairs.  (Few rows, one chunk
    and several; many rows, alone and with their keys split.)"""
    Lq, Lk, H, Hk, D = shape
    x, _ = draw(5, Lq, Lk, H, Hk, D, dtype)
    clean = {n: t.clone() for n, t in x.items()}
    lens = torch.tensor([Lk, Lk, Lk, 0, Lk], dtype=torch.int32)
    x["q"][1, Lq - 1, H - 1] = math.nan
    x["k"][2, 0, Hk - 1, 3] = math.nan     # every query of those heads sees it, the first one only it (not align_end)
    x["k"][4] = math.nan
    x["q"][3, 0] = math.nan                # no pair: nothing to see
    opts = {"causal": True, "align_end": end}
    res = []
    for y in (clean, x):
        res.append(pkg.seq_attention_forward(*(y[n].cuda() for n in "qkv"), kv_len=lens.cuda(), **opts))
    bad = nan_rows(x, lens, **opts)
    assert bad.any() and not bad[3].any()
    (out0, lse0), (out, lse) = [(o.cpu(), l.cpu()) for o, l in res]
    rows = bad.transpose(1, 2)
    assert torch.equal(torch.isnan(lse), bad)
    assert torch.isnan(out[rows]).all()
    assert torch.equal(out[~rows], out0[~rows]) and torch.equal(lse[~bad], lse0[~bad])
    assert (out[3] == 0).all() and (lse[3] == -math.inf).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("cap", [200.0, 300.0, 1e4, 1e6])
def test_large_caps(cap, dtype):
    """Scores far below their cap.  There tanh(u) is its series, whose error is
    relative to u: the reference's allowance of 4 roundings of the cap falls
    away (but for 16 bits up to 256, where it is below a sixteenth of P's own
    rounding), the 8 of a score cover the products with scale/cap, cap*log2(e)
    and the series' own."""
    for causal in (False, True):
        x, _ = draw(2, 90, 90, 2, 2, 64, dtype, seed=int(cap))
        opts = {"cap": cap, "causal": causal}
        ref = Attention(x["q"], x["k"], x["v"], **opts)
        assert float(ref.t.abs().max()) < 0.25
        if dtype == F32 or cap > 256:
            ref.e -= 2.0 ** -24 * 4 * cap
        q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
        out, lse = pkg.seq_attention_forward(q, k, v, **opts)
        to, tl = ref.tolerances()
        check(out, ref.out.transpose(1, 2), to + 1e-30, "out")
        check(lse, ref.lse, tl + 1e-30, "lse")
        # one dout row at a time: a sum over many rows hides what one is off by
        for rows in (slice(0, 90), slice(3, 4), slice(60, 61)):
            x1 = torch.zeros_like(x["dout"])
            x1[:, rows] = x["dout"][:, rows]
            grads = pkg.seq_attention_backward(x1.cuda(), q, k, v, out, lse, **opts)
            want, tol = ref.grads(x1, out.cpu(), lse.cpu())
            for name, a, w, t in zip(("dq", "dk", "dv"), grads, want, tol):
                check(a, w, t, name)


@pytest.mark.parametrize("types", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)], ids=ids)
@pytest.mark.parametrize("C", [40, 1025, 16384, 20000, 33001])
def test_layer_norm_without_rows(C, types):
    """No rows: gradients of zero, for rows that fit the registers and longer ones."""
    dt, wdt = types
    x = torch.zeros((0, C), dtype=dt, device="cuda")
    w = torch.ones(C, dtype=wdt, device="cuda")
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w, w)
    assert y.shape == (0, C)
    dx, dw, db = pkg.seq_layer_norm_backward(x, x, w, mean, rstd)
    assert dx.shape == (0, C) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("types", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)], ids=ids)
@pytest.mark.parametrize("size", [(2, 32768), (3, 32776), (5, 33001)], ids=str)
def test_layer_norm_long_rows(size, types):
    """The longest rows that 16-bit types hold in registers, and longer."""
    layer_norm_case(size, types)


def forward_and_backward(x, bias, opts):
    o = {k: to_gpu(v) for k, v in opts.items()}
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    out, lse = pkg.seq_attention_forward(q, k, v, bias=to_gpu(bias), **o)
    return (out, lse) + tuple(pkg.seq_attention_backward(do, q, k, v, out, lse, bias=to_gpu(bias), **o))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("hold", [math.nan, math.inf, -math.inf], ids=str)
@pytest.mark.parametrize("Lq,Lk", [(100, 128), (33, 64), (70, 600), (1, 40)])
def test_keys_behind_the_last_query(Lq, Lk, hold, dtype):
    """Causal, more keys than queries: the keys that no query sees have no
    influence and gradients of zero, also beside the padding of a query tile."""
    x, bias = draw(2, Lq, Lk, 2, 1, 64, dtype, R=10)
    res = []
    for value in (0.0, hold):
        y = {n: t.clone() for n, t in x.items()}
        y["k"][:, Lq:] = value
        y["v"][:, Lq:] = value
        res.append(forward_and_backward(y, bias, {"causal": True}))
    for a, b in zip(*res):
        assert not torch.isnan(b).any() and torch.equal(a, b)
    assert (res[1][3][:, Lq:] == 0).all() and (res[1][4][:, Lq:] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("hold", [math.nan, math.inf], ids=str)
def test_keys_of_documents_without_queries(hold, dtype):
    """Keys of document 0 where no query has it; the padding of a query tile has none either."""
    B, Lq, Lk = 2, 100, 150
    x, bias = draw(B, Lq, Lk, 2, 2, 64, dtype, R=10)
    g = torch.Generator().manual_seed(1)
    q_doc = torch.randint(1, 3, (B, Lq), generator=g).to(torch.int32)
    k_doc = torch.randint(0, 3, (B, Lk), generator=g).to(torch.int32)
    q_doc[1] = 1
    k_doc[1] = 0
    res = []
    for value in (0.0, hold):
        y = {n: t.clone() for n, t in x.items()}
        y["k"][k_doc == 0] = value
        y["v"][k_doc == 0] = value
        res.append(forward_and_backward(y, bias, {"q_doc": q_doc, "k_doc": k_doc}))
    for a, b in zip(*res):
        assert not torch.isnan(b).any() and torch.equal(a, b)
    gone = (k_doc == 0).cuda()
    assert (res[1][3][gone] == 0).all() and (res[1][4][gone] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_keys_of_minus_infinity(dtype):
    """Keys whose scores are -inf for every query have probability 0: dv, dk
    and the strip's gradient are those of keys far away, whatever the padding
    of a query tile makes of them."""
    x, bias = draw(1, 100, 100, 2, 2, 64, dtype, R=10)
    x["q"] = x["q"].abs() + 0.5
    res = []
    for value in (-6e4, -math.inf):
        y = {n: t.clone() for n, t in x.items()}
        y["k"][0, 40] = value
        res.append(forward_and_backward(y, bias, {}))
    for n in (0, 1, 3, 4, 5):
        assert torch.equal(res[0][n], res[1][n]), n


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("masks", ["causal", "prefix", "align_end", "documents", "causal documents", "lengths"])
def test_largest_numbers_in_keys_and_values_nobody_sees(masks, dtype):
    """The type's largest number where no query looks: nothing changes, fp16's
    scale of the gradients neither."""
    big = torch.finfo(dtype).max
    B, Lq, Lk = 2, 100, 230
    g = torch.Generator().manual_seed(2)
    j = torch.arange(Lk)[None].expand(B, Lk)
    opts = {"causal": {"causal": True}, "prefix": {"causal": True, "prefix": torch.tensor([150, 3], dtype=torch.int32)},
            "align_end": {"causal": True, "align_end": True, "kv_len": torch.tensor([230, 120], dtype=torch.int32)},
            "lengths": {"kv_len": torch.tensor([130, 7], dtype=torch.int32)}}.get(masks, {"causal": masks[0] == "c"})
    if "documents" in masks:
        qd = torch.randint(-1, 3, (B, Lq), generator=g)     # any order; document 3 has no query
        kd = torch.randint(-1, 4, (B, Lk), generator=g)
        qd[1] = torch.arange(Lq) // 33 * 2                  # runs: 0, 2, 4, 6; 1, 3, 5 have no query
        kd[1] = torch.arange(Lk) // 40
        opts.update(q_doc=qd.to(torch.int32), k_doc=kd.to(torch.int32))
    x, bias = draw(B, Lq, Lk, 2, 1, 64, dtype, R=10)
    seen = allowed(B, Lq, Lk, **opts)[0].any(1)
    assert not seen.all()
    res = []
    for value in (0.0, big):
        y = {n: t.clone() for n, t in x.items()}
        y["k"][~seen] = value
        y["v"][~seen] = value
        res.append(forward_and_backward(y, bias, opts))
    for a, b in zip(*res):
        assert not torch.isnan(b).any() and torch.equal(a, b)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (BF16, BF16)], ids=ids)
@pytest.mark.parametrize("C", [5, 100])
def test_layer_norm_huge_constant_rows(C, types):
    """Rows of one value near the type's largest: x - mean is 0, though
    mean*rstd is beyond the range; lanes beyond the row add nothing."""
    dt, wdt = types
    x = torch.full((3, C), 2.0 ** 120, dtype=dt, device="cuda")     # sums of up to 100 are exact and finite
    g = torch.Generator().manual_seed(C)
    dy = torch.randn((3, C), generator=g).to(dt)
    w = (torch.randn(C, generator=g) + 1).to(wdt)
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w.cuda(), w.cuda())
    assert torch.equal(mean.cpu(), torch.full((3,), 2.0 ** 120)) and torch.equal(y.cpu(), w.to(dt).expand(3, C))
    dx, dw, db = pkg.seq_layer_norm_backward(dy.cuda(), x, w.cuda(), mean, rstd)
    G, rs = dy.double() * w.double(), rstd.double().cpu()[:, None]
    want = rs * (G - G.mean(1, keepdim=True))
    u = 2.0 ** -8 if dt == BF16 else 2.0 ** -24
    check(dx, want, 2.0 ** -24 * 64 * rs * (G.abs() + G.abs().mean(1, keepdim=True)) + u * want.abs(), "dx")
    assert (dw == 0).all()
    check(db, dy.double().sum(0), (2.0 ** -22 + (2.0 ** -8 if wdt == BF16 else 0)) * dy.double().abs().sum(0), "db")


def busy(n=4):
    """Some 25 ms of work on the current stream."""
    a = torch.ones((8192, 8192), device="cuda")
    for _ in range(n):
        a @ a


def stream_calls():
    x = torch.randn((2048, 512), device="cuda")
    w, b = torch.rand(512, device="cuda"), torch.randn(512, device="cuda")
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w, b)
    table = torch.randn((32, 64), device="cuda")
    ds = torch.randn((8, 64, 2049), device="cuda")
    q = torch.randn((2, 1024, 8, 64), device="cuda").to(BF16)
    k, v = torch.randn_like(q), torch.randn_like(q)
    out, lse = pkg.seq_attention_forward(q, k, v)
    return {
        "layer norm": (pkg.seq_layer_norm_forward, (x, w, b)),
        "layer norm backward": (pkg.seq_layer_norm_backward, (y, x, w, mean, rstd)),
        "bias": (pkg.seq_rel_bias_forward, (table, 1024)),
        "bias backward": (pkg.seq_rel_bias_backward, (ds, 32)),
        "attention": (pkg.seq_attention_forward, (q, k, v)),
        "attention backward": (pkg.seq_attention_backward, (out, q, k, v, out, lse)),
    }


@pytest.mark.parametrize("name", ["layer norm", "layer norm backward", "bias", "bias backward", "attention",
                                  "attention backward"])
@pytest.mark.parametrize("handle", [False, True], ids=["stream", "handle"])
def test_memory_of_calls_on_another_stream(name, handle):
    """A block freed here while work that reads it is pending is not written
    by a call on another stream; a tensor given to such a call and freed is
    not reused before it has been read."""
    fn, args = stream_calls()[name]
    want = fn(*args)
    want = [t for t in (want if isinstance(want, tuple) else (want,)) if t is not None]
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    # blocks of the results' sizes, freed while copies from them are pending
    held = [torch.full_like(t, 7) for t in want]
    to = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    busy()
    for t, h in zip(to, held):
        t.copy_(h)
    del held, h
    got = fn(*args, stream=stream)
    side.synchronize()
    torch.cuda.synchronize()
    for t in to:
        assert (t == 7).all()
    got = [t for t in (got if isinstance(got, tuple) else (got,)) if t is not None]
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # inputs freed while the call waits behind other work of its stream
    args = tuple(t.clone() if isinstance(t, torch.Tensor) else t for t in args)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    got = fn(*args, stream=stream)
    sizes = [t.shape for t in args if isinstance(t, torch.Tensor)], [t.dtype for t in args if isinstance(t, torch.Tensor)]
    del args
    over = [torch.full(s, math.nan, dtype=d, device="cuda") for s, d in zip(*sizes)]
    torch.cuda.synchronize()
    got = [t for t in (got if isinstance(got, tuple) else (got,)) if t is not None]
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_the_null_stream_by_its_handle():
    x = torch.randn((64, 512), device="cuda")
    w = torch.rand(512, device="cuda")
    want = pkg.seq_layer_norm_forward(x, w, w)
    torch.cuda.synchronize()
    got = pkg.seq_layer_norm_forward(x, w, w, stream=0)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Lq", [1, 33])
def test_strip_offsets_beyond_32_bits(Lq):
    """So many heads that the last ones' bias lies more than 2^31 floats behind
    the first's; more heads, too, than a grid has in its second dimension."""
    H, R, L, D = 1048100, 1024, 33, 8
    assert (H - 20) * (2 * R + 1) > 2 ** 31
    part = torch.arange(H - 3, H)                     # the heads that are looked at, and the first
    part = torch.cat([torch.tensor([0, 65535, 65536]), part])
    g = torch.Generator().manual_seed(Lq)
    small = {n: torch.randn((1, Lq if n in ("q", "dout") else L, len(part), D), generator=g).to(F16)
             for n in ("q", "k", "v", "dout")}
    strip = torch.randn((len(part), 2 * R + 1), generator=g)
    x = {n: torch.zeros((1, t.shape[1], H, D), dtype=F16, device="cuda") for n, t in small.items()}
    for n, t in small.items():
        x[n][:, :, part.cuda()] = t.cuda()
    bias = torch.zeros((H, 2 * R + 1), device="cuda")
    for i, h in enumerate(part.tolist()):
        bias[h] = strip[i].cuda()
    ref = Attention(small["q"], small["k"], small["v"], bias=strip)
    out, lse = pkg.seq_attention_forward(x["q"], x["k"], x["v"], bias=bias)
    to, tl = ref.tolerances()
    pick = part.cuda()
    check(out[:, :, pick], ref.out.transpose(1, 2), to + 1e-30, "out")
    check(lse[:, pick], ref.lse, tl + 1e-30, "lse")
    grads = pkg.seq_attention_backward(x["dout"], x["q"], x["k"], x["v"], out, lse, bias=bias)
    want, tol = ref.grads(small["dout"], out[:, :, pick].cpu(), lse[:, pick].cpu())
    for name, a, w, t in zip(("dq", "dk", "dv"), grads, want, tol):
        check(a[:, :, pick], w, t, name)
    check(torch.stack([grads[3][h] for h in part.tolist()]), want[3], tol[3], "dstrip")


PACKED = {  # order in memory of sequences 0, tokens 1, heads 2, parts (q, k, v) 3, channels 4
    "parts within tokens": (0, 1, 3, 2, 4),
    "sequences within tokens": (1, 0, 3, 2, 4),
    "heads before tokens": (0, 3, 2, 1, 4),
    "parts within heads": (0, 1, 2, 3, 4),
}


def packed_like(B, L, H, D, order, dtype):
    """([B][L][H][D] views x 3 of one tensor whose dimensions lie in `order`, that tensor)"""
    dims = (B, L, H, 3, D)
    t = torch.full([dims[d] for d in order], 7, dtype=dtype, device="cuda")
    back = [order.index(d) for d in range(5)]
    return t.permute(back).unbind(3), t


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("layout", sorted(PACKED))
def test_packed_layouts(layout, dtype):
    """q, k and v in one tensor, and their gradients in another, in any order of its dimensions."""
    B, L, H, D = 3, 70, 2, 64
    x, bias = draw(B, L, L, H, H, D, dtype, R=7)
    want = forward_and_backward(x, bias, {"causal": True})
    (q, k, v), _ = packed_like(B, L, H, D, PACKED[layout], dtype)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        t.copy_(x[n])
    (dq, dk, dv), whole = packed_like(B, L, H, D, PACKED[layout], dtype)
    out, lse = pkg.seq_attention_forward(q, k, v, bias=bias.cuda(), causal=True, out=dq)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert (dk == 7).all() and (dv == 7).all()
    out = out.clone()
    got = pkg.seq_attention_backward(x["dout"].cuda(), q, k, v, out, lse, bias=bias.cuda(), causal=True, dq=dq, dk=dk, dv=dv)
    for a, b in zip(got, want[2:]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("layout", sorted(PACKED))
def test_packed_layouts_that_meet(layout):
    """The same layouts moved so that two outputs share bytes."""
    B, L, H, D = 3, 20, 2, 64
    x, _ = draw(B, L, L, H, H, D, F16)
    q, k, v, do = (x[n].cuda() for n in ("q", "k", "v", "dout"))
    out, lse = pkg.seq_attention_forward(q, k, v)
    (dq, dk, dv), whole = packed_like(B, L, H, D, PACKED[layout], F16)
    flat = torch.zeros(whole.numel() + 64, dtype=F16, device="cuda")
    for shift in (8, 32, 56):
        at = dk.storage_offset() + shift
        moved = flat.as_strided(dk.shape, dk.stride(), at)
        first = flat.as_strided(dq.shape, dq.stride(), dq.storage_offset())
        last = flat.as_strided(dv.shape, dv.stride(), dv.storage_offset())
        with pytest.raises(pkg.Im2winError) as e:
            pkg.seq_attention_backward(do, q, k, v, out, lse, dq=first, dk=moved, dv=last)
        assert e.value.status == -7


def test_one_token_beside_the_keys():
    """The output of a single token in a row that keys and values lie in."""
    B, L, H, D = 1, 50, 2, 64
    whole = torch.randn((B, L, 3, H, D), device="cuda")
    k, v = whole[:, :, 0], whole[:, :, 1]
    q = torch.randn((B, 1, H, D), device="cuda")
    want, _ = pkg.seq_attention_forward(q, k.contiguous(), v.contiguous())
    before = whole.clone()
    out, _ = pkg.seq_attention_forward(q, k, v, out=whole[:, 7:8, 2])
    assert torch.equal(out, want) and torch.equal(whole[:, :, :2], before[:, :, :2])
    with pytest.raises(pkg.Im2winError):
        pkg.seq_attention_forward(q, k, v, out=whole[:, 7:8, 1])


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_strides_of_dimensions_of_one(dtype):
    """The stride of a dimension with one element is not a step: any value will do."""
    B, H, D = 2, 2, 64
    x, bias = draw(B, 1, 1, H, H, D, dtype, R=7)
    want = forward_and_backward(x, bias, {})
    far = {n: t.cuda().as_strided(t.shape, (H * D, 1 << 40, D, 1)) for n, t in x.items()}
    new = [torch.empty((B, 1, H, D), dtype=dtype, device="cuda").as_strided((B, 1, H, D), (H * D, 12345, D, 1)) for _ in range(4)]
    out, lse = pkg.seq_attention_forward(far["q"], far["k"], far["v"], bias=bias.cuda(), out=new[0])
    got = pkg.seq_attention_backward(far["dout"], far["q"], far["k"], far["v"], out, lse, bias=bias.cuda(), dq=new[1],
                                     dk=new[2], dv=new[3])
    for a, b in zip((out, lse) + got, want):
        assert torch.equal(a, b)
    # one sequence, one head
    x, bias = draw(1, 40, 70, 1, 1, D, dtype, R=7)
    want = forward_and_backward(x, bias, {})
    far = {n: t.cuda().as_strided(t.shape, (1 << 50, D, (1 << 45) + 3, 1)) for n, t in x.items()}
    for a, b in zip(forward_and_backward(x, bias, {}), want):
        assert torch.equal(a, b)
    out, lse = pkg.seq_attention_forward(far["q"], far["k"], far["v"], bias=bias.cuda())
    got = pkg.seq_attention_backward(far["dout"], far["q"], far["k"], far["v"], out, lse, bias=bias.cuda())
    for a, b in zip((out, lse) + got, want):
        assert torch.equal(a, b)


def test_sequences_far_apart():
    """Sequences more than 2^32 elements from each other, as in a cache of many layers."""
    L, D, step = 40, 64, (1 << 32) + 64
    x, _ = draw(2, L, L, 1, 1, D, F16)
    want = forward_and_backward(x, None, {})
    big = torch.empty(step + 2 * L * D, dtype=F16, device="cuda")
    k = big.as_strided((2, L, 1, D), (step, D, D, 1))
    v = big[L * D:].as_strided((2, L, 1, D), (step, D, D, 1))
    k.copy_(x["k"])
    v.copy_(x["v"])
    q, do = x["q"].cuda(), x["dout"].cuda()
    out, lse = pkg.seq_attention_forward(q, k, v)
    for a, b in zip((out, lse) + tuple(pkg.seq_attention_backward(do, q, k, v, out, lse))[:3], want):
        assert torch.equal(a, b)


def test_layer_norm_rows_far_apart():
    """Rows more than 2^29 elements from each other."""
    step, C = (1 << 30) + 8, 200
    big = torch.empty(step + 2 * C, dtype=F16, device="cuda")
    x, dy = big.as_strided((2, C), (step, 1)), big[C:].as_strided((2, C), (step, 1))
    g = torch.Generator().manual_seed(4)
    for t in (x, dy):
        t.copy_(torch.randn((2, C), generator=g))
    w = torch.rand(C, generator=g).cuda()
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w, w)
    want = pkg.seq_layer_norm_forward(x.contiguous(), w, w)
    got = (y, mean, rstd) + pkg.seq_layer_norm_backward(dy, x, w, mean, rstd)
    for a, b in zip(got, want + pkg.seq_layer_norm_backward(dy.contiguous(), x.contiguous(), w, mean, rstd)):
        assert torch.equal(a, b)


MASKS = {
    "none": {},
    "causal cap": {"causal": True, "cap": 20.0},
    "lengths at the end": {"causal": True, "align_end": True, "lens": True},
    "lengths": {"lens": True},
    "documents": {"docs": True},
    "causal documents cap": {"causal": True, "docs": True, "cap": 20.0, "lens": True},
    "prefix": {"causal": True, "prefix": True},
}


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("masks", sorted(MASKS))
@pytest.mark.parametrize("shape", [(2, 130, 700, 3, 1, 80), (3, 200, 1100, 4, 2, 64), (1, 65, 1300, 2, 2, 128),
                                   (2, 300, 600, 2, 1, 32)], ids=str)
def test_keys_shared_by_workgroups(shape, masks, dtype):
    """Rows long enough, and few enough, that their keys are split over
    workgroups and the parts joined, forward (512 keys on in fp32, 1024 in 16
    bits) and backward (256, 512); masks under which some parts have no key,
    with and without a bias."""
    B, Lq, Lk, H, Hk, D = shape
    g = torch.Generator().manual_seed(Lk + len(masks))
    opts = dict(MASKS[masks])
    if opts.pop("lens", False):
        opts["kv_len"] = torch.tensor([Lk, 0, Lk // 3][:B], dtype=torch.int32)
    if opts.pop("prefix", False):
        opts["prefix"] = torch.tensor([Lk - 5, 0, 70][:B], dtype=torch.int32)
    if opts.pop("docs", False):
        kd = (torch.arange(Lk)[None] // torch.tensor([[90], [40], [333]][:B])).to(torch.int32)
        kd[:, -20:] = -1
        opts["q_doc"], opts["k_doc"] = kd[:, :Lq].clone(), kd
        opts["q_doc"][0] = torch.randint(-1, 8, (Lq,), generator=g)
    x, bias = draw(*shape, dtype, seed=Lk, R=90)
    run(x, None, opts)
    run(x, bias, opts)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("hold", [math.nan, math.inf, -math.inf, "largest"], ids=str)
@pytest.mark.parametrize("cap", [5.0, 1000.0])
def test_masked_places_with_a_cap(cap, hold, dtype):
    """What masked places hold has no influence on capped scores either: the
    slope of a left-out score may be NaN.  Masks that cut through tiles, with
    and without a bias."""
    hold = torch.finfo(dtype).max if hold == "largest" else hold
    B, Lq, Lk = 3, 100, 150
    doc = torch.arange(Lk)[None].expand(B, Lk) // torch.tensor([[50], [9], [200]])
    doc = torch.where(torch.arange(Lk)[None] % 7 == 3, torch.full_like(doc, -1), doc).to(torch.int32)
    for opts in ({"causal": True, "align_end": True, "kv_len": torch.tensor([Lk, 77, 0], dtype=torch.int32)},
                 {"causal": True}, {"q_doc": doc[:, :Lq].contiguous(), "k_doc": doc}):
        x, bias = draw(B, Lq, Lk, 2, 1, 64, dtype, R=10)
        ok = allowed(B, Lq, Lk, **opts)[0]
        for strip in (None, bias):
            res = []
            for value in (0.0, hold):
                y = {n: t.clone() for n, t in x.items()}
                for n, seen in (("q", ok.any(2)), ("dout", ok.any(2)), ("k", ok.any(1)), ("v", ok.any(1))):
                    y[n][~seen] = value
                res.append(forward_and_backward(y, strip, {**opts, "cap": cap}))
            for a, b in zip(*res):
                assert a is None or (not torch.isnan(b).any() and torch.equal(a, b))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_a_key_that_is_nan_reaches_only_its_pairs(dtype):
    """Gradients beside a NaN key, capped: NaN in the queries that see it, not in the others of its tile."""
    L = 100
    x, _ = draw(1, L, L, 1, 1, 64, dtype)
    x["k"][0, 40] = math.nan
    for cap in (0.0, 5.0, 1000.0):
        res = forward_and_backward(x, None, {"causal": True, "cap": cap})
        out, lse, dq = res[0].cpu(), res[1].cpu(), res[2].cpu()
        assert torch.isfinite(out[0, :40]).all() and torch.isfinite(lse[0, 0, :40]).all() and torch.isfinite(dq[0, :40]).all()
        assert torch.isnan(out[0, 40:]).all() and torch.isnan(lse[0, 0, 40:]).all() and torch.isnan(dq[0, 40:]).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("hold", [math.nan, math.inf], ids=str)
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_dv_takes_what_is_not_finite_from_dout_alone(cap, hold, dtype):
    """dv = P^T dout: a value that is not finite does not reach it, a dout
    only the channel it stands in, also in tiles with left-out pairs."""
    L = 100
    x, _ = draw(1, L, L, 2, 1, 64, dtype)
    opts = {"causal": True, "cap": cap}
    clean = forward_and_backward(x, None, opts)
    y = {n: t.clone() for n, t in x.items()}
    y["v"][0, 20, 0, 5] = hold
    assert torch.equal(forward_and_backward(y, None, opts)[4], clean[4])
    y = {n: t.clone() for n, t in x.items()}
    y["dout"][0, 70, 1, 5] = hold
    dv = forward_and_backward(y, None, opts)[4]
    want = torch.zeros((1, L, 1, 64), dtype=torch.bool)
    want[0, :71, 0, 5] = True
    assert torch.equal(~torch.isfinite(dv.cpu()), want)
    same = ~want.cuda()
    assert torch.equal(dv[same], clean[4][same])
