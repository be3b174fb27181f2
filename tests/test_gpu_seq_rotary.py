"""Rotary positions against the formulas in 64 bits: types, both orders of
pairs, parts of heads, strides, positions, in place, gradients, streams and
graphs."""
import pytest
import torch

import paper_2608_20725_amd as pkg
from gpu_util import say
from seq_cache_ref import rotary
from seq_ref import check

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def inputs(B, L, H, D, dtype, seed=0, far=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, L, H, D), generator=g).to(dtype)
    first = torch.randint(0, far + 1, (B, 1), generator=g)
    return x, (first + torch.arange(L)).int()


# tokens and heads on both sides of the rule for heads a lane; whole heads and
# parts; parts that end inside a vector, odd halves, one pair; odd tails
SHAPES = [(1, 1, 1, 2, 2), (4, 1, 40, 128, 128), (2, 37, 5, 80, 40), (3, 50, 3, 96, 50), (2, 9, 4, 64, 2), (2, 70, 7, 33, 22),
          (1, 5, 2, 256, 256), (2, 33, 2, 300, 254), (2, 1100, 40, 128, 128), (1, 3001, 13, 72, 48), (2, 1500, 11, 130, 98)]


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_backward(shape, dtype, interleaved):
    B, L, H, D, rot = shape
    say("rotary", shape, dtype, interleaved)
    x, pos = inputs(B, L, H, D, dtype, far=100000)
    freq = pkg.seq_rotary_frequencies(rot, factor=4.0, trained=4096)
    for fn, back in ((pkg.seq_rotary_forward, False), (pkg.seq_rotary_backward, True)):
        got = fn(x.cuda(), freq, pos.cuda(), interleaved=interleaved, amplitude=1.25)
        want, tol = rotary(x, freq.tolist(), pos, interleaved, 1.25, back)
        bare = tol == 0
        check(got, want, torch.where(bare, torch.ones_like(tol), tol), "rotary")
        assert torch.equal(got.cpu()[bare], x[bare])


@pytest.mark.parametrize("at", [0, 1, -1, 4096, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31])
def test_far_positions(at):
    """Angles of any int32 position, frequencies from 1 to 1e-6 and the largest
    allowed ones."""
    x, _ = inputs(1, 3, 2, 64, torch.float32)
    pos = torch.tensor([[at, 0, 7]], dtype=torch.int32)
    for freq in (pkg.seq_rotary_frequencies(64, base=1e6), torch.linspace(-1024, 1024, 32, dtype=torch.float64)):
        got = pkg.seq_rotary_forward(x.cuda(), freq, pos.cuda())
        want, tol = rotary(x, freq.tolist(), pos)
        check(got, want, tol, "far")


def test_positions_by_sequence_and_none():
    x, _ = inputs(3, 41, 4, 64, torch.float32)
    freq = pkg.seq_rotary_frequencies(64)
    first = torch.tensor([0, 5000, 2 ** 31 - 20], dtype=torch.int32)  # runs on past 2^31
    t = torch.arange(41)
    got = pkg.seq_rotary_forward(x.cuda(), freq, first.cuda())
    want, tol = rotary(x, freq.tolist(), first[:, None].long() + t)
    check(got, want, tol, "by sequence")
    got = pkg.seq_rotary_forward(x.cuda(), freq)
    want, tol = rotary(x, freq.tolist(), t.expand(3, 41))
    check(got, want, tol, "none")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_and_in_place(dtype, interleaved):
    """Columns of a packed tensor, heads first, rows that start anywhere; the
    tensor itself; what lies beside is left alone."""
    x, pos = inputs(2, 35, 6, 48, dtype, far=9)
    freq = pkg.seq_rotary_frequencies(40)
    want, tol = rotary(x, freq.tolist(), pos, interleaved)
    tol = tol + 1e-30
    wide = torch.full((2, 35, 9, 51), float("nan"), dtype=dtype, device="cuda")
    packed = wide[:, :, 2:8, 1:49]
    packed.copy_(x)
    first = x.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    for src in (packed, first):
        check(pkg.seq_rotary_forward(src, freq, pos.cuda(), interleaved), want, tol, "strided")
        assert torch.equal(src.cpu(), x)
    out = torch.full((6, 2, 35, 50), float("nan"), dtype=dtype, device="cuda").permute(1, 2, 0, 3)
    assert pkg.seq_rotary_forward(packed, freq, pos.cuda(), interleaved, out=out[..., 1:49]).data_ptr() == out[..., 1:].data_ptr()
    check(out[..., 1:49], want, tol, "out")
    assert torch.isnan(out[..., 0]).all() and torch.isnan(out[..., 49]).all()
    pkg.seq_rotary_forward(packed, freq, pos.cuda(), interleaved, out=packed)
    check(packed, want, tol, "in place")
    packed.fill_(float("nan"))
    assert torch.isnan(wide).all()
    many = x[:, :, :1].cuda().expand(2, 35, 6, 48)  # one head read as six
    w1, t1 = rotary(x[:, :, :1].expand(2, 35, 6, 48), freq.tolist(), pos, interleaved)
    check(pkg.seq_rotary_forward(many, freq, pos.cuda(), interleaved), w1, t1 + 1e-30, "expanded")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
@pytest.mark.parametrize("shape", [(2, 1500, 12, 60, 50), (2, 1500, 12, 128, 38), (3, 3000, 5, 24, 14), (2, 31, 3, 24, 14),
                                   (1, 20000, 8, 40, 2), (2, 9000, 8, 26, 26), (1, 3, 2, 10, 6)], ids=lambda s: "x".join(map(str, s)))
def test_in_place_where_units_overlap(shape, dtype, interleaved):
    """Pairs that no unit divides: the last unit takes pairs of the one before
    again, which in place may be turned already.  The same bits both ways."""
    B, L, H, D, rot = shape
    x, pos = inputs(B, L, H, D, dtype, far=77)
    freq = pkg.seq_rotary_frequencies(rot)
    xd, pd = x.cuda(), pos.cuda()
    want = pkg.seq_rotary_forward(xd, freq, pd, interleaved)
    ref, tol = rotary(x[:, :40], freq.tolist(), pos[:, :40], interleaved)
    bare = tol == 0
    check(want[:, :40], ref, torch.where(bare, torch.ones_like(tol), tol), "rotary")
    for _ in range(3):
        again = xd.clone()
        pkg.seq_rotary_forward(again, freq, pd, interleaved, out=again)
        assert torch.equal(again, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "pairs"])
@pytest.mark.parametrize("D,rot", [(64, 2), (64, 6), (64, 20), (64, 60), (72, 32), (80, 80), (30, 22)])
def test_long_calls_are_short_ones_in_a_row(D, rot, dtype, interleaved):
    """Bit for bit, though lanes take more pairs and heads; copied channels as they are."""
    B, L, H = 2, 2100, 27
    x, pos = inputs(B, L, H, D, dtype, seed=3, far=9000)
    freq = pkg.seq_rotary_frequencies(rot)
    xd, pd = x.cuda(), pos.cuda()
    xd[:, ::7, :, rot:] = float("nan")
    got = pkg.seq_rotary_forward(xd, freq, pd, interleaved)
    for at in (0, 1000, 2095):
        few = slice(at, at + 5)
        want = pkg.seq_rotary_forward(xd[:, few], freq, pd[:, few].contiguous(), interleaved)
        assert torch.equal(got[:, few, :, :rot], want[..., :rot])
    bits = {4: torch.int32, 2: torch.int16}[x.element_size()]
    assert torch.equal(got[..., rot:].contiguous().view(bits), xd[..., rot:].contiguous().view(bits))
    ref, tol = rotary(x[:, 1000:1040], freq.tolist(), pos[:, 1000:1040], interleaved)
    check(got[:, 1000:1040, :, :rot], ref[..., :rot], tol[..., :rot], "rotary")
    pkg.seq_rotary_forward(xd, freq, pd, interleaved, out=xd)
    assert torch.equal(xd[..., :rot], got[..., :rot])


def test_gradient_against_differences():
    """sum(dy * y(x + h d)) - sum(dy * y(x - h d)) over 2h against sum(dx * d):
    the map is linear, so the difference is exact but for rounding (fp32, sums
    of 2*9*3*32 products of size 1: 2^-24 * 2 * 1728 / (2h) at most)."""
    x, pos = inputs(2, 9, 3, 32, torch.float32, seed=1, far=1000)
    d, dy = (inputs(2, 9, 3, 32, torch.float32, seed=s)[0] for s in (2, 3))
    freq = pkg.seq_rotary_frequencies(24)
    f = lambda v: pkg.seq_rotary_forward(v.cuda(), freq, pos.cuda(), amplitude=0.7).double().cpu()
    diff = float((dy.double() * (f(x + d) - f(x - d))).sum() / 2)
    dx = pkg.seq_rotary_backward(dy.cuda(), freq, pos.cuda(), amplitude=0.7).double().cpu()
    assert abs(diff - float((dx * d.double()).sum())) <= 2.0 ** -24 * 8 * 1728


def test_values_that_are_not_finite_stay_in_their_pair():
    x, pos = inputs(1, 4, 2, 16, torch.float32)
    freq = pkg.seq_rotary_frequencies(8)
    clean = pkg.seq_rotary_forward(x.cuda(), freq, pos.cuda()).cpu()
    bad = x.clone()
    bad[0, 1, 0, 2], bad[0, 2, 1, 12] = float("nan"), float("inf")
    got = pkg.seq_rotary_forward(bad.cuda(), freq, pos.cuda()).cpu()
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[0, 1, 0, 2] = hit[0, 1, 0, 6] = hit[0, 2, 1, 12] = True
    assert torch.equal(got[~hit], clean[~hit])
    assert torch.isnan(got[0, 1, 0, 2]) and torch.isnan(got[0, 1, 0, 6]) and torch.isinf(got[0, 2, 1, 12])


def test_refusals():
    x = torch.zeros(2, 4, 3, 16, device="cuda")
    freq = pkg.seq_rotary_frequencies(16)

    def status(*a, **k):
        with pytest.raises(pkg.Im2winError) as e:
            pkg.seq_rotary_forward(*a, **k)
        return e.value.status
    wide = torch.zeros(2, 5, 3, 16, device="cuda")
    assert status(wide[:, :4], freq, out=wide[:, 1:]) == -7
    assert status(x, freq, out=x[:, :, :1].expand(2, 4, 3, 16)) == -7       # an output onto itself
    assert status(x[:, :, :1].expand(2, 4, 3, 16), freq, out=x) == -7       # in place needs the same strides
    ints = torch.zeros(392, dtype=torch.int32, device="cuda")               # positions inside the output
    assert status(x, freq, ints[:8].view(2, 4), out=ints[4:388].view(torch.float32).view(2, 4, 3, 16)) == -7
    assert status(x.cpu(), freq) == -8


def test_empty():
    freq = pkg.seq_rotary_frequencies(16)
    for shape in ((0, 4, 3, 16), (2, 0, 3, 16), (2, 4, 0, 16)):
        assert pkg.seq_rotary_forward(torch.zeros(shape, device="cuda"), freq).shape == shape


def test_another_stream_and_graph():
    x, pos = inputs(2, 33, 8, 64, torch.bfloat16, far=50)
    freq = pkg.seq_rotary_frequencies(64)
    xd, pd = x.cuda(), pos.cuda()
    want = pkg.seq_rotary_forward(xd, freq, pd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = pkg.seq_rotary_forward(xd, freq, pd, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(xd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.seq_rotary_forward(xd, freq, pd, out=out)
    del freq  # its values travelled with the call
    for k in range(3):
        xd.copy_(x.cuda() * (k + 1))
        pd.add_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = pkg.seq_rotary_forward(xd, pkg.seq_rotary_frequencies(64), pd)
        assert torch.equal(out, again), k
