"""Layer norm and the relative position bias against the plain form in 64 bits."""
import math

import pytest
import torch

import paper_2608_20725_amd as pkg
from seq_ref import U, bucket, check

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)]
ids = lambda v: str(v).replace("torch.", "")

# rows, C: lane-held rows of one and four waves at both ends of every size class, odd and unaligned, the looped kernels
SIZES = [(1, 1), (1, 2), (5, 3), (3, 64), (7, 65), (33, 127), (4, 128), (9, 256), (2, 512), (5, 771), (3, 1000), (70, 1024),
         (3, 1025), (2, 2048), (3, 2056), (2, 4096), (2, 4104), (3, 5001), (2, 8192), (2, 8200), (1, 8193), (2, 16384),
         (1, 20000), (130, 96)]


def norm_ref(x, w, b, eps):
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + eps)
    return mean, rstd, (x - mean) * rstd * w + b


@pytest.mark.parametrize("types", TYPES, ids=ids)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_layer_norm(size, types):
    rows, C = size
    dt, wdt = types
    g = torch.Generator().manual_seed(rows * 131 + C)
    for pad, eps in ((0, 1e-5), (5, 0.1)):
        wide = (torch.randn((rows, C + pad), generator=g) * (torch.rand((rows, 1), generator=g) + 0.1)
                + 3 * torch.randn((rows, 1), generator=g)).to(dt)
        dyw = torch.randn((rows, C + pad), generator=g).to(dt)
        x, dy = wide[:, :C], dyw[:, :C]
        w, b = (torch.randn(C, generator=g) + 1).to(wdt), torch.randn(C, generator=g).to(wdt)
        xd, dyd = wide.cuda()[:, :C], dyw.cuda()[:, :C]
        y, mean, rstd = pkg.seq_layer_norm_forward(xd, w.cuda(), b.cuda(), eps)
        X, W, Bb = x.double(), w.double(), b.double()
        m, r, ref = norm_ref(X, W, Bb, eps)
        # fp32 sums of C terms: mean off by e*max|x|, the variance by 2 e of
        # itself plus that squared, where e = 2^-24 (log2 of the lanes' tree
        # and 32 terms a lane; C/256 for the looped rows)
        e = 2.0 ** -24 * (48 + C / 256)
        big = X.abs().amax(1, keepdim=True) + 1e-30
        tm = e * big
        tr = r * (4 * e + (tm * r) ** 2 + 2 * tm * r * (C == 1))
        check(mean, m[:, 0], tm[:, 0], "mean")
        check(rstd, r[:, 0], tr[:, 0] + 1e-30, "rstd")
        ty = (tm * r + (X - m).abs() * tr + 4 * 2.0 ** -24 * (X - m).abs() * r) * W.abs() + U[dt] * ref.abs() \
            + 2.0 ** -23 * (ref.abs() + Bb.abs()) + (6e-8 if dt == F16 else 1e-30)
        check(y, ref, ty, "y")
        # backward, from the statistics the forward call gave
        dx, dw, db = pkg.seq_layer_norm_backward(dyd, xd, w.cuda(), mean, rstd)
        mu, rs = mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
        h, G, DY = (X - mu) * rs, dy.double() * W, dy.double()
        want = rs * (G - G.mean(1, keepdim=True) - h * (G * h).mean(1, keepdim=True))
        he = 4 * 2.0 ** -24 * (X.abs() + mu.abs()) * rs                   # error of h
        size_ = G.abs() + G.abs().mean(1, keepdim=True) + h.abs() * (G * h).abs().mean(1, keepdim=True)
        tx = rs * (4 * e * size_ + he * (G * h).abs().mean(1, keepdim=True) + h.abs() * (G.abs() * he).mean(1, keepdim=True)) \
            + U[dt] * want.abs() + (6e-8 if dt == F16 else 1e-30)
        check(dx, want, tx, "dx")
        n = 2.0 ** -24 * (rows + 40)
        dW, dB = (DY * h).sum(0), DY.sum(0)
        check(dw, dW, n * (DY * h).abs().sum(0) + (DY.abs() * he).sum(0) + U[wdt] * dW.abs() + (6e-8 if wdt == F16 else 1e-30), "dw")
        check(db, dB, n * DY.abs().sum(0) + U[wdt] * dB.abs() + (6e-8 if wdt == F16 else 1e-30), "db")


@pytest.mark.parametrize("rows", [1000, 40000])
def test_layer_norm_many_rows(rows):
    """More rows than workgroups: every row once, sums over all."""
    C = 96
    x = torch.randn((rows, C), device="cuda")
    w, b = torch.rand(C, device="cuda") + 0.5, torch.randn(C, device="cuda")
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w, b)
    X = x.double()
    m, r, ref = norm_ref(X, w.double(), b.double(), 1e-5)
    assert float((y.double() - ref).abs().max()) < 1e-4
    dy = torch.randn_like(x)
    dx, dw, db = pkg.seq_layer_norm_backward(dy, x, w, mean, rstd)
    h = (X - mean.double()[:, None]) * rstd.double()[:, None]
    n = 2.0 ** -24 * (rows + 40)
    assert ((dw.double() - (dy.double() * h).sum(0)).abs() <= (n + 1e-6) * (dy.double() * h).abs().sum(0)).all()
    assert ((db.double() - dy.double().sum(0)).abs() <= n * dy.double().abs().sum(0)).all()
    again = pkg.seq_layer_norm_backward(dy, x, w, mean, rstd)
    for p, q in zip((dx, dw, db), again):
        assert torch.equal(p, q)


def test_layer_norm_shapes_and_views():
    x = torch.randn((2, 3, 5, 40), device="cuda")
    w, b = torch.rand(40, device="cuda"), torch.randn(40, device="cuda")
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w, b)
    assert y.shape == x.shape and mean.shape == (2, 3, 5)
    y2, _, _ = pkg.seq_layer_norm_forward(x.view(30, 40), w, b)
    assert torch.equal(y.view(30, 40), y2)
    x2 = x.clone()
    y3, _, _ = pkg.seq_layer_norm_forward(x2, w, b, out=x2)      # in place
    assert y3 is x2 and torch.equal(y3, y)
    # unaligned views: one element off
    flat = torch.randn(1 + 30 * 40, device="cuda", dtype=F32).to(F16)
    v = flat[1:].view(30, 40)
    a, _, _ = pkg.seq_layer_norm_forward(v, w.to(F16), b.to(F16))
    c, _, _ = pkg.seq_layer_norm_forward(v.clone(), w.to(F16), b.to(F16))
    assert float((a.float() - c.float()).abs().max()) <= 2.0 ** -8
    e = torch.zeros((0, 40), device="cuda")
    y, mean, rstd = pkg.seq_layer_norm_forward(e, w, b)
    assert y.shape == (0, 40)
    dx, dw, db = pkg.seq_layer_norm_backward(e, e, w, mean, rstd)
    assert (dw == 0).all() and (db == 0).all()


def test_layer_norm_large_offset_and_not_finite():
    x = torch.randn((4, 640), device="cuda") + 1e4           # the centred sum keeps the variance
    w, b = torch.ones(640, device="cuda"), torch.zeros(640, device="cuda")
    x[1, 5], x[2, 7] = math.nan, math.inf
    y, mean, rstd = pkg.seq_layer_norm_forward(x, w, b)
    for r in (0, 3):
        m, s, ref = norm_ref(x[r:r + 1].double(), w.double(), b.double(), 1e-5)
        assert float((y[r].double() - ref[0]).abs().max()) < 2.0 ** -24 * 1e4 * 64
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).any()


BIAS = [(8, 5, True), (8, 5, False), (32, 128, True), (32, 128, False), (320, 800, True), (64, 40, True), (512, 1024, False),
        (4, 1024, True), (2, 2, False), (1024, 1024, True)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=ids)
@pytest.mark.parametrize("plan", BIAS, ids=str)
def test_rel_bias(plan, dtype):
    nb, R, two = plan
    for H, n in ((1, 1), (5, 3)):
        g = torch.Generator().manual_seed(nb + H)
        table = torch.randn((nb, H), generator=g).to(dtype)
        at = torch.tensor([bucket(d, nb, R, two) for d in range(-R, R + 1)])
        strip = pkg.seq_rel_bias_forward(table.cuda(), R, two_sided=two)
        assert torch.equal(strip.cpu(), table.float()[at].t())
        ds = torch.randn((n, H, 2 * R + 1), generator=g)
        dt = pkg.seq_rel_bias_backward(ds.cuda(), nb, two_sided=two, dtype=dtype)
        want = torch.zeros((nb, H), dtype=torch.float64).index_add_(0, at, ds.double().sum(0).t())
        size = torch.zeros((nb, H), dtype=torch.float64).index_add_(0, at, ds.double().abs().sum(0).t())
        check(dt, want, 2.0 ** -24 * (n * R / 16 + 40) * size + U[dtype] * want.abs() + 1e-30
              + (6e-8 if dtype == F16 else 0), "dtable")
        if n == 1:
            assert torch.equal(pkg.seq_rel_bias_backward(ds[0].cuda(), nb, two_sided=two, dtype=dtype), dt)
