"""The sequence operators whose speed counts: layer norm, relative position bias and attention.

A case is one pass through an operator as a program makes it: ``ln_fwd`` / ``ln_bwd`` normalise rows of channels
(pixels or tokens), ``bias_fwd`` / ``bias_bwd`` take a learned table of distance buckets to the strip that attention
reads and the strips' gradients back to the table's, ``attn_fwd`` / ``attn_bwd`` are attention over a batch of token
rows with its masks, cap and bias, and ``decode`` is attention of a few new tokens over a long cache.  With ``own``
false every operator is computed from elementary torch operations in 32 bits; with ``own`` true by the framework.

Fields: ``dt`` element type; layer norm: ``rows``, ``C``, ``pad`` (elements between rows beyond C), ``wdt`` type of
weight and bias; bias: ``H`` heads, ``nb`` buckets, ``R`` largest distance, ``two`` two-sided, ``n`` layers that share
the table; attention: B, Lq, Lk, H, Hk (key/value heads), D, ``causal``, ``end`` (queries are the last positions),
``cap`` (0: none), ``nb``/``R``/``two`` (R 0: no bias), ``docs`` (documents in a row, 0: no document mask), ``prefix``
(share of the row all queries see, in percent), ``ragged`` (sequences of different lengths).
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-5


def _ln(name, op, dt, rows, C, pad=0, wdt=None):
    return {"name": name, "op": op, "dt": dt, "rows": rows, "C": C, "pad": pad, "wdt": wdt or dt}


def _bias(name, op, H, nb, R, two=True, n=1, dt="f32"):
    return {"name": name, "op": op, "dt": dt, "H": H, "nb": nb, "R": R, "two": two, "n": n}


def _attn(name, op, dt, B, Lq, Lk, H, Hk, D, causal=False, end=False, cap=0.0, nb=0, R=0, two=True, docs=0, prefix=0,
          ragged=False):
    return {"name": name, "op": op, "dt": dt, "B": B, "Lq": Lq, "Lk": Lk, "H": H, "Hk": Hk, "D": D, "causal": causal,
            "end": end, "cap": cap, "nb": nb, "R": R, "two": two, "docs": docs, "prefix": prefix, "ragged": ragged}


def listed():
    return [
        # one step of token generation for four sequences: latency only
        _ln("ln_4_tokens_bf16", "ln_fwd", "bf16", 4, 1024),
        # rows cut out of a wider tensor, odd channel count, fp32
        _ln("ln_ragged_f32", "ln_fwd", "f32", 9765, 771, pad=29),
        # training over the pixels of a stage: 128 images of 28x28, 512 channels, fp32 weights
        _ln("ln_train_bf16", "ln_bwd", "bf16", 100352, 512, wdt="f32"),
        # the strip of a small encoder, made once a step
        _bias("bias_strip_32_f32", "bias_fwd", 16, 32, 128),
        # the table's gradient from the 24 layers that share it, wide range as in audio encoders
        _bias("bias_grad_24_layers", "bias_bwd", 16, 320, 800, n=24),
        # image encoder: 14x14 tokens, small heads, learned bias
        _attn("attn_196_bias_f16", "attn_fwd", "f16", 8, 196, 196, 8, 8, 64, nb=32, R=128),
        # packed pretraining rows: documents, causal, capped scores, shared key/value heads
        _attn("attn_8k_docs_cap_bf16", "attn_fwd", "bf16", 2, 8192, 8192, 16, 4, 128, causal=True, cap=50.0, docs=7),
        # prefix-LM scoring in fp32, odd lengths, head size that is no power of two
        _attn("attn_prefix_1001_f32", "attn_fwd", "f32", 3, 1001, 1001, 6, 6, 80, causal=True, prefix=30, ragged=True),
        # encoder training on 28x28 tokens padded to the longest, bias with its gradient
        _attn("attn_train_784_bias_f16", "attn_bwd", "f16", 16, 784, 784, 16, 16, 64, nb=32, R=128, ragged=True),
        # the largest: decoder training, long rows, shared heads, capped scores
        _attn("attn_train_4k_cap_bf16", "attn_bwd", "bf16", 2, 4096, 4096, 32, 8, 128, causal=True, cap=30.0),
        # chat with one user: one new token, a cache of some thousand, bias
        _attn("decode_1x2000_bias_f16", "decode", "f16", 1, 1, 2000, 16, 4, 64, causal=True, end=True, nb=32, R=128,
              two=False),
        # serving: 32 sequences of up to 8192 tokens, one new token each
        _attn("decode_32x8k_bf16", "decode", "bf16", 32, 1, 8192, 32, 8, 128, causal=True, end=True, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _clean(n):
    return n + 1 if n == 3072 else n


def draw(rng):
    """One more case: any operator, type, mask and length of the listed ranges."""
    op = rng.choice(["ln_fwd", "ln_bwd", "bias_fwd", "bias_bwd", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd", "decode",
                     "decode"])
    dt = rng.choice(["f32", "f16", "bf16"])
    if op in ("ln_fwd", "ln_bwd"):
        C = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            C = max(16, C // 8 * 8)
        rows = _log_int(rng, 1, max(2, 51380224 // C))
        return _ln(None, op, dt, _clean(rows), _clean(C), pad=rng.choice([0, 0, 8, rng.randint(1, 64)]),
                   wdt=rng.choice([dt, "f32"])) | {"name": ""}
    if op in ("bias_fwd", "bias_bwd"):
        two = rng.random() < 0.5
        nb = 2 * _log_int(rng, 4, 160)
        return _bias("", op, rng.randint(1, 64), nb, nb + _log_int(rng, 1, 700), two=two,
                     n=1 if op == "bias_fwd" else _log_int(rng, 1, 24), dt=dt)
    D = rng.choice([32, 64, 64, 80, 96, 128, 128, 8 * rng.randint(1, 16)])
    Hk = rng.choice([1, 2, 4, 8])
    H = Hk * rng.choice([1, 1, 2, 3, 4, 8])
    nb, R, two = (0, 0, True) if rng.random() < 0.5 else (32, rng.randint(40, 800), rng.random() < 0.5)
    cap = rng.choice([0.0, 0.0, 30.0, 50.0])
    if op == "decode":
        B, Lk = _log_int(rng, 1, 32), _log_int(rng, 64, 8192)
        return _attn("", op, dt, B, rng.choice([1, 1, 2, 5]), _clean(Lk), min(H, 32), min(Hk, min(H, 32)), D, causal=True, end=True,
                     cap=cap, nb=nb, R=R, two=two, ragged=rng.random() < 0.7)
    L = _clean(_log_int(rng, 16, 8192 if op == "attn_fwd" else 4096))
    cross = rng.random() < 0.2
    Lk = _clean(_log_int(rng, 16, 4096)) if cross else L
    # f32 runs at a sixteenth of the 16-bit rate
    most = (2 if dt == "f32" else 12) * 2 ** 26
    B = max(1, min(_log_int(rng, 1, 64), most // (H * L * Lk)))
    causal = not cross and rng.random() < 0.6
    return _attn("", op, dt, B, L, Lk, H, Hk, D, causal=causal, cap=cap, nb=nb, R=R, two=two,
                 docs=0 if cross or rng.random() < 0.6 else rng.randint(1, 12),
                 prefix=rng.randint(5, 60) if causal and rng.random() < 0.3 else 0, ragged=rng.random() < 0.4)


# ---- what belongs to a case's shape: lengths, documents, prefixes -------------------------------------------------

def _lens(c):
    """Key count of each sequence (all Lk where the case is not ragged): from a quarter of Lk to Lk."""
    if not c["ragged"]:
        return [c["Lk"]] * c["B"]
    lo = max(1, c["Lk"] // 4)
    return [c["Lk"]] + [lo + (b * 7919 * 13) % (c["Lk"] - lo + 1) for b in range(1, c["B"])]


def _docs(c):
    """Document id of every position, documents of uneven length, the last 2 % of a row padding (-1)."""
    L, n = c["Lk"], c["docs"]
    rows = []
    for b in range(c["B"]):
        used = L - L // 50
        cuts = sorted({(used * (k * k + b * k)) // (n * n + b * n) for k in range(1, n)} | {used})
        ids, at = [], 0
        for k, e in enumerate(cuts):
            ids += [k] * (e - at)
            at = e
        rows.append(ids + [-1] * (L - used))
    return rows


def _prefix(c):
    return [max(1, c["Lk"] * c["prefix"] // 100) // (1 + b % 3) for b in range(c["B"])]


def _masks(c, device):
    """The mask's inputs as device arrays, None where the case has none."""
    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=device)
    return {"kv_len": ints(_lens(c)) if c["ragged"] else None, "prefix": ints(_prefix(c)) if c["prefix"] else None,
            "doc": ints(_docs(c)) if c["docs"] else None}


def _allowed(c, m, b, device):
    """[Lq][Lk] truth values of sequence b: the pairs that take part."""
    n = c["Lk"] if m["kv_len"] is None else m["kv_len"][b]
    i = torch.arange(c["Lq"], device=device)[:, None]
    j = torch.arange(c["Lk"], device=device)[None, :]
    p = i + (n - c["Lq"]) if c["end"] else i
    ok = (j < n).expand(c["Lq"], c["Lk"])
    if c["causal"]:
        see = j <= p
        if m["prefix"] is not None:
            see = see | (j < m["prefix"][b])
        ok = ok & see
    if m["doc"] is not None:
        d = m["doc"][b]
        ok = ok & (d[:, None] == d[None, :]) & (d >= 0)[:, None]
    return ok, j - p


def _first(c, b):
    """Distance of key 0 from query 0."""
    return c["Lq"] - _lens(c)[b] if c["end"] else 0


# ---- inputs ------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(dev).manual_seed(int(seed))
    dt = _DT[c["dt"]]

    def normal(*shape, dtype=dt, mean=0.0, std=1.0):
        return (torch.randn(shape, generator=g, device=dev) * std + mean).to(dtype)

    s = {"case": c}
    if c["op"] in ("ln_fwd", "ln_bwd"):
        rows, C, wdt = c["rows"], c["C"], _DT[c["wdt"]]
        # activations: a row has its own offset and scale
        wide = torch.randn((rows, C + c["pad"]), generator=g, device=dev)
        off = torch.randn((rows, 1), generator=g, device=dev)
        size = torch.rand((rows, 1), generator=g, device=dev) * 2 + 0.25
        s["x"] = (wide * size + off).to(dt)[:, :C]
        s["w"], s["b"] = normal(C, dtype=wdt, mean=1.0, std=0.2), normal(C, dtype=wdt, std=0.2)
        if c["op"] == "ln_bwd":
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = ((x - s["mean"][:, None]).square().mean(1) + _EPS).rsqrt()
            s["dy"] = normal(rows, C)
        return s
    if c["op"] == "bias_fwd":
        s["table"] = normal(c["nb"], c["H"])
        return s
    if c["op"] == "bias_bwd":
        s["dstrip"] = normal(c["n"], c["H"], 2 * c["R"] + 1, dtype=torch.float32)
        return s
    B, Lq, Lk, H, Hk, D = (c[k] for k in ("B", "Lq", "Lk", "H", "Hk", "D"))
    if Lq == Lk and H == Hk:   # the projection's output: q, k and v side by side in each token's row
        s["q"], s["k"], s["v"] = normal(B, Lq, 3, H, D).unbind(2)
    else:
        s["q"], s["k"], s["v"] = normal(B, Lq, H, D), normal(B, Lk, Hk, D), normal(B, Lk, Hk, D)
    s.update(_masks(c, dev))
    if c["R"]:
        s["table"] = normal(c["nb"], H, dtype=torch.float32)
    if c["op"] == "attn_bwd":
        s["out"], s["lse"] = _attention(s)
        s["dout"] = normal(B, Lq, H, D)
    if c["R"] and c["op"] != "attn_fwd":
        # serving makes the strip once, a training step has it from its forward pass
        s["strip"] = _strip(s["table"], c)
    return s


# ---- plain forms: elementary operations in 32 bits ---------------------------------------------------------------

def _bucket(c, device):
    """Bucket of every distance -R .. R (key position minus query position)."""
    d = torch.arange(-c["R"], c["R"] + 1, device=device)
    m = c["nb"] // 2 if c["two"] else c["nb"]
    e = m // 2
    n = d.abs() if c["two"] else (-d).clamp(min=0)
    far = torch.floor(torch.log(n.clamp(min=e).double() / e) / math.log(c["R"] / e) * (m - e) + 1e-9).long() + e
    b = torch.where(n < e, n, far.clamp(max=m - 1))
    return b + m * (d > 0) if c["two"] else b


def _strip(table, c):
    return table.float()[_bucket(c, table.device)].t().contiguous()


def _table_grad(by_distance, c, first):
    """[nb][H] from sums [H][T] of the distances first, first + 1, ..: each bucket's summed."""
    dev = by_distance.device
    d = torch.arange(first, first + by_distance.shape[1], device=dev).clamp(-c["R"], c["R"])
    one = torch.zeros((d.numel(), c["nb"]), device=dev)
    one[torch.arange(d.numel(), device=dev), _bucket(c, dev)[d + c["R"]]] = 1
    return (by_distance @ one).t().contiguous()


def _diagonals(x):
    """Sums of [H][Lq][Lk] over its diagonals, [H][Lq + Lk - 1] by key minus query from 1 - Lq on: rows of the upside
    down matrix padded to Lq + Lk and read one element shorter put each diagonal into one column."""
    H, Lq, Lk = x.shape
    wide = torch.nn.functional.pad(x.flip(1), (0, Lq)).reshape(H, -1)
    return wide[:, :Lq * (Lq + Lk - 1)].view(H, Lq, Lq + Lk - 1).sum(1)


def _scores(s, b, strip):
    """Scores [H][Lq][Lk] of sequence b (masked pairs -inf), the capped part over the cap, and the mask."""
    c = s["case"]
    G = c["H"] // c["Hk"]
    q = s["q"][b].float().transpose(0, 1).contiguous()
    k = s["k"][b].float().permute(1, 2, 0).contiguous().repeat_interleave(G, 0)
    x = torch.bmm(q, k) * (c["D"] ** -0.5)
    t = None
    if c["cap"]:
        t = torch.tanh(x / c["cap"])
        x = t * c["cap"]
    ok, d = _allowed(c, s, b, q.device)
    if c["R"]:
        x = x + strip[:, d.clamp(-c["R"], c["R"]) + c["R"]]
    return x.masked_fill(~ok, float("-inf")), t, ok


def _attention(s, strip=None):
    c = s["case"]
    G = c["H"] // c["Hk"]
    if c["R"] and strip is None:
        strip = _strip(s["table"], c)
    outs, lses = [], []
    for b in range(c["B"]):
        x, _, _ = _scores(s, b, strip)
        top = x.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        e = torch.exp(x - top)
        z = e.sum(-1, keepdim=True)
        v = s["v"][b].float().transpose(0, 1).contiguous().repeat_interleave(G, 0)
        o = torch.bmm(e, v) / torch.where(z > 0, z, torch.ones_like(z))
        outs.append(o.transpose(0, 1))
        lses.append((torch.log(z) + top)[..., 0])
    return torch.stack(outs).to(_DT[c["dt"]]), torch.stack(lses)


def _attention_grad(s):
    c = s["case"]
    dt, G, H = _DT[c["dt"]], c["H"] // c["Hk"], c["H"]
    strip = s.get("strip")
    dqs, dks, dvs = [], [], []
    dtable = torch.zeros((c["nb"], H), device=s["q"].device)
    for b in range(c["B"]):
        x, t, ok = _scores(s, b, strip)
        lse = s["lse"][b][..., None]
        p = torch.where(ok, torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)), torch.zeros_like(x))
        do = s["dout"][b].float().transpose(0, 1).contiguous()
        vt = s["v"][b].float().permute(1, 2, 0).contiguous().repeat_interleave(G, 0)
        delta = (do * s["out"][b].float().transpose(0, 1)).sum(-1, keepdim=True)
        ds = p * (torch.bmm(do, vt) - delta)
        if c["R"]:
            dtable += _table_grad(_diagonals(ds), c, 1 - c["Lq"] + _first(c, b))
        if t is not None:
            ds = ds * (1 - t * t)
        ds = ds * (c["D"] ** -0.5)
        q = s["q"][b].float().transpose(0, 1).contiguous()
        k = s["k"][b].float().transpose(0, 1).contiguous().repeat_interleave(G, 0)
        dq = torch.bmm(ds, k)
        dk = torch.bmm(ds.transpose(1, 2).contiguous(), q).view(c["Hk"], G, c["Lk"], c["D"]).sum(1)
        dv = torch.bmm(p.transpose(1, 2).contiguous(), do).view(c["Hk"], G, c["Lk"], c["D"]).sum(1)
        dqs.append(dq.transpose(0, 1))
        dks.append(dk.transpose(0, 1))
        dvs.append(dv.transpose(0, 1))
    grads = [torch.stack(g).to(dt) for g in (dqs, dks, dvs)]
    return grads + ([dtable] if c["R"] else [])


def _plain(s):
    c = s["case"]
    if c["op"] == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = ((x - mean).square().mean(1, keepdim=True) + _EPS).rsqrt()
        y = (x - mean) * rstd * s["w"].float() + s["b"].float()
        return [y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]]
    if c["op"] == "ln_bwd":
        dy, mean, rstd = s["dy"].float(), s["mean"][:, None], s["rstd"][:, None]
        xh = (s["x"].float() - mean) * rstd
        g = dy * s["w"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return [dx.to(s["x"].dtype), (dy * xh).sum(0).to(s["w"].dtype), dy.sum(0).to(s["w"].dtype)]
    if c["op"] == "bias_fwd":
        return [_strip(s["table"], c)]
    if c["op"] == "bias_bwd":
        return [_table_grad(s["dstrip"].sum(0), c, -c["R"]).to(_DT[c["dt"]])]
    if c["op"] == "attn_bwd":
        return _attention_grad(s)
    return list(_attention(s, s.get("strip")))


# ---- the framework's operators -----------------------------------------------------------------------------------

def _own(s):
    import paper_2608_20725_amd as im2win
    c = s["case"]
    if c["op"] == "ln_fwd":
        return list(im2win.seq_layer_norm_forward(s["x"], s["w"], s["b"], _EPS))
    if c["op"] == "ln_bwd":
        return list(im2win.seq_layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"]))
    if c["op"] == "bias_fwd":
        return [im2win.seq_rel_bias_forward(s["table"], c["R"], two_sided=c["two"])]
    if c["op"] == "bias_bwd":
        return [im2win.seq_rel_bias_backward(s["dstrip"], c["nb"], two_sided=c["two"], dtype=_DT[c["dt"]])]
    opts = dict(cap=c["cap"], causal=c["causal"], align_end=c["end"], kv_len=s["kv_len"], prefix=s["prefix"],
                q_doc=s["doc"], k_doc=s["doc"])
    if c["op"] == "attn_bwd":
        dq, dk, dv, dstrip = im2win.seq_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"],
                                                           bias=s.get("strip"), **opts)
        if not c["R"]:
            return [dq, dk, dv]
        return [dq, dk, dv, im2win.seq_rel_bias_backward(dstrip, c["nb"], two_sided=c["two"], dtype=torch.float32)]
    strip = s.get("strip")
    if c["R"] and strip is None:
        strip = im2win.seq_rel_bias_forward(s["table"], c["R"], two_sided=c["two"])
    return list(im2win.seq_attention_forward(s["q"], s["k"], s["v"], bias=strip, **opts))


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def _pairs(c):
    m = _masks(c, "cpu")
    total = 0
    for b in range(c["B"]):
        if c["docs"] or c["prefix"]:
            total += int(_allowed(c, m, b, "cpu")[0].sum())
            continue
        n, Lq = _lens(c)[b], c["Lq"]
        if not c["causal"]:
            total += n * Lq
            continue
        off = n - Lq if c["end"] else 0
        total += sum(max(0, min(n, i + off + 1)) for i in range(Lq))
    return total


def work(case):
    c = case
    size = {"f32": 4, "f16": 2, "bf16": 2}
    e = size[c["dt"]]
    if c["op"] == "ln_fwd":
        n = c["rows"] * c["C"]
        return {"bytes": 2 * n * e + 2 * c["C"] * size[c["wdt"]] + 8 * c["rows"], "flops": 8 * n}
    if c["op"] == "ln_bwd":
        n = c["rows"] * c["C"]
        return {"bytes": 3 * n * e + 3 * c["C"] * size[c["wdt"]] + 8 * c["rows"], "flops": 14 * n}
    if c["op"] in ("bias_fwd", "bias_bwd"):
        n = c["n"] * c["H"] * (2 * c["R"] + 1)
        return {"bytes": 4 * n + c["nb"] * c["H"] * e, "flops": n}
    keys = sum(_lens(c))
    q, kv, rows = c["B"] * c["Lq"] * c["H"] * c["D"] * e, 2 * keys * c["Hk"] * c["D"] * e, c["B"] * c["H"] * c["Lq"]
    if c["op"] == "attn_bwd":   # q, out, dout, k, v, lse in; dq, dk, dv out
        kv_out = 2 * c["B"] * c["Lk"] * c["Hk"] * c["D"] * e
        return {"bytes": 4 * q + kv + kv_out + 4 * rows, "flops": 10 * _pairs(c) * c["H"] * c["D"]}
    return {"bytes": 2 * q + kv + 4 * rows, "flops": 4 * _pairs(c) * c["H"] * c["D"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _exact_bucket(c):
    """Bucket of distance d, one at a time, from the definition."""
    out = []
    for d in range(-c["R"], c["R"] + 1):
        m, first = (c["nb"] // 2, c["nb"] // 2 if d > 0 else 0) if c["two"] else (c["nb"], 0)
        n, e = (abs(d) if c["two"] else max(0, -d)), m // 2
        if n < e:
            out.append(first + n)
        else:
            out.append(first + min(m - 1, e + math.floor(math.log(n / e) / math.log(c["R"] / e) * (m - e) + 1e-9)))
    return out


def _exact_attention(s):
    c = s["case"]
    H, Hk, D, Lq, Lk, R = c["H"], c["Hk"], c["D"], c["Lq"], c["Lk"], c["R"]
    grad = c["op"] == "attn_bwd"
    dev, f64 = s["q"].device, torch.float64
    out, lse = torch.zeros((c["B"], Lq, H, D), dtype=f64, device=dev), torch.zeros((c["B"], H, Lq), dtype=f64, device=dev)
    dq = torch.zeros_like(out)
    dk = torch.zeros((c["B"], Lk, Hk, D), dtype=f64, device=dev)
    dv = torch.zeros_like(dk)
    if R:
        bucket = torch.tensor(_exact_bucket(c), device=dev)
        if grad or c["op"] == "decode":
            strip = s["strip"].double()
        else:
            strip = s["table"].double()[bucket].t()
        dtable = torch.zeros((c["nb"], H), dtype=f64, device=dev)
    for b in range(c["B"]):
        ok, d = _allowed(c, s, b, dev)
        d = d.clamp(-R, R) + R
        for h in range(H):
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :, h * Hk // H].double(), s["v"][b, :, h * Hk // H].double()
            z = q @ k.t() / math.sqrt(D)
            slope = 1.0
            if c["cap"]:
                th = torch.tanh(z / c["cap"])
                z, slope = c["cap"] * th, 1 - th ** 2
            if R:
                z = z + strip[h][d]
            z = torch.where(ok, z, torch.full_like(z, -math.inf))
            if not grad:
                lse[b, h] = torch.logsumexp(z, 1)
                out[b, :, h] = torch.where(ok.any(1, keepdim=True), torch.softmax(z, 1), torch.zeros_like(z)) @ v
                continue
            l = s["lse"][b, h].double()[:, None]
            p = torch.where(ok & torch.isfinite(l), (z - l).exp(), torch.zeros_like(z))
            do, o = s["dout"][b, :, h].double(), s["out"][b, :, h].double()
            dz = p * (do @ v.t() - (do * o).sum(1, keepdim=True))
            if R:
                dtable[:, h].index_add_(0, bucket[d].reshape(-1), dz.reshape(-1))
            dz = dz * slope / math.sqrt(D)
            dq[b, :, h] = dz @ k
            dk[b, :, h * Hk // H] += dz.t() @ q
            dv[b, :, h * Hk // H] += p.t() @ do
    if not grad:
        return [out, lse]
    return [dq, dk, dv] + ([dtable] if R else [])


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "ln_fwd":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1 / torch.sqrt(var + _EPS)
        return [(x - mean[:, None]) * rstd[:, None] * s["w"].double() + s["b"].double(), mean, rstd]
    if c["op"] == "ln_bwd":
        dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
        xh = (s["x"].double() - s["mean"].double()[:, None]) * rstd
        g = dy * s["w"].double()
        dx = rstd * (g - (g.sum(1, keepdim=True) + xh * (g * xh).sum(1, keepdim=True)) / c["C"])
        return [dx, (dy * xh).sum(0), dy.sum(0)]
    if c["op"] == "bias_fwd":
        return [s["table"].double()[torch.tensor(_exact_bucket(c), device=s["table"].device)].t()]
    if c["op"] == "bias_bwd":
        d = s["dstrip"].double().sum(0)
        out = torch.zeros((c["nb"], c["H"]), dtype=torch.float64, device=d.device)
        return [out.index_add_(0, torch.tensor(_exact_bucket(c), device=d.device), d.t())]
    return _exact_attention(s)
