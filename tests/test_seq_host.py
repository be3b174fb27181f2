"""The sequence operators' C interface on the host: the library exports what
im2win_seq.h declares, refuses what the header rules out, and its host-only
functions do what the header states.  No call here reaches a GPU."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2608_20725_amd as pkg
from paper_2608_20725_amd import seq
from seq_ref import bucket

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "im2win_seq.h")
EINVAL, EALIGN, ERANGE, EWORKSPACE, EOVERLAP = -1, -2, -3, -6, -7
P = 1 << 40  # an aligned address nothing is read from


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.library_path()):
        from paper_2608_20725_amd import build
        build.build()
    return seq._library()


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return set(re.findall(r"\b(seq_\w+)\s*\(", text))


def test_library_exports_what_the_header_declares(lib):
    out = subprocess.run(["nm", "-D", "--defined-only", pkg.library_path()], capture_output=True, text=True, check=True)
    exported = {l.split()[-1] for l in out.stdout.splitlines() if " T " in l}
    assert {n for n in exported if n.startswith("seq_")} == declared()


def test_header_is_c():
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", "-x", "c", HEADER], check=True)


def test_description_has_the_structs_size(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "im2win_seq.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) { printf("%zu %zu %zu %zu", '
                   'sizeof(seq_attention_t), offsetof(seq_attention_t, B), offsetof(seq_attention_t, R), '
                   'offsetof(seq_attention_t, k_doc)); return 0; }\n')
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    size, b, r, kd = map(int, subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split())
    assert seq._PACK.size == size
    packed = seq._PACK.pack(*([0] * 3), 0.0, 0.0, 77, *([0] * 29), 78, *([0] * 4), 79)
    assert int.from_bytes(packed[b:b + 8], "little") == 77
    assert int.from_bytes(packed[r:r + 8], "little") == 78
    assert int.from_bytes(packed[kd:kd + 8], "little") == 79


@pytest.mark.parametrize("nb,R,two", [(32, 128, True), (32, 128, False), (2, 2, False), (4, 1024, True), (512, 1024, False),
                                      (320, 800, True), (1024, 1024, True), (8, 5, False)])
def test_buckets(lib, nb, R, two):
    for d in list(range(-R - 3, R + 4)) + [-10 ** 6, 10 ** 6]:
        assert pkg.seq_rel_bias_bucket(d, nb, R, two) == bucket(d, nb, R, two), d


@pytest.mark.parametrize("nb,R,two,status", [(0, 8, True, EINVAL), (7, 8, True, EINVAL), (2, 8, True, EINVAL),
                                             (32, 8, True, EINVAL), (32, 16, False, EINVAL), (32, 0, True, EINVAL),
                                             (32, 1025, True, ERANGE), (514, 1000, False, ERANGE)])
def test_bucket_plans_refused(lib, nb, R, two, status):
    assert lib.seq_rel_bias_bucket(0, nb, R, int(two)) == status
    assert lib.seq_rel_bias_forward(P, 2 * P, 4, nb, R, int(two), 0, None) == status
    assert lib.seq_rel_bias_backward(P, 2 * P, 1, 4, nb, R, int(two), 0, None) == status


def test_rel_bias_refusals(lib):
    f, b = lib.seq_rel_bias_forward, lib.seq_rel_bias_backward
    assert f(None, P, 4, 32, 128, 1, 0, None) == EINVAL
    assert f(P, None, 4, 32, 128, 1, 0, None) == EINVAL
    assert f(P, 2 * P, 4, 32, 128, 1, 3, None) == EINVAL
    assert f(P, 2 * P, 0, 32, 128, 1, 0, None) == EINVAL
    assert f(P, 2 * P, 1 << 16, 32, 128, 1, 0, None) == ERANGE
    assert f(P + 2, 2 * P, 4, 32, 128, 1, 0, None) == EALIGN
    assert f(P, 2 * P + 2, 4, 32, 128, 1, 1, None) == EALIGN
    assert b(P, 2 * P, -1, 4, 32, 128, 1, 0, None) == EINVAL
    assert b(P, 2 * P, 1 << 16, 4, 32, 128, 1, 0, None) == ERANGE
    assert b(None, 2 * P, 1, 4, 32, 128, 1, 0, None) == EINVAL


def norm_forward(lib, x=P, w=2 * P, b=3 * P, y=4 * P, mean=5 * P, rstd=6 * P, rows=4, C=8, xs=8, eps=1e-5, dt=0, wdt=0):
    return lib.seq_layer_norm_forward(x, w, b, y, mean, rstd, rows, C, xs, eps, dt, wdt, None)


def test_layer_norm_refusals(lib):
    f = lambda **k: norm_forward(lib, **k)
    for k in ({"x": None}, {"w": None}, {"b": None}, {"y": None}, {"mean": None}, {"rstd": None}, {"rows": -1}, {"C": 0},
              {"xs": 7}, {"eps": -1.0}, {"eps": float("nan")}, {"dt": 3}, {"dt": 0, "wdt": 1}, {"dt": 1, "wdt": 2}):
        assert f(**k) == EINVAL, k
    assert f(C=1 << 24, xs=1 << 24) == ERANGE
    assert f(rows=1 << 31) == ERANGE
    assert f(x=P + 2) == EALIGN and f(dt=1, wdt=1, x=P + 1) == EALIGN and f(mean=5 * P + 2) == EALIGN
    assert f(rows=0, x=None, y=None, mean=None, rstd=None) == 0     # nothing to do, before any device is asked
    ws = lib.seq_layer_norm_workspace_bytes
    assert ws(-1, 4) == EINVAL and ws(4, 0) == EINVAL and ws(1 << 31, 4) == ERANGE and ws(4, 1 << 24) == ERANGE
    assert ws(0, 5) > 0 and ws(1000, 512) >= 1000 // 32 * 2 * 512 * 4
    back = lambda *a: lib.seq_layer_norm_backward(*a, None)
    good = [P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 7 * P, 8 * P, 9 * P, 1 << 20, 4, 8, 8, 8, 0, 0]
    for i in range(9):
        bad = list(good)
        bad[i] = None
        assert back(*bad) == EINVAL
    bad = list(good)
    bad[9] = -1
    assert back(*bad) == EWORKSPACE
    bad = list(good)
    bad[8] = 9 * P + 8
    assert back(*bad) == EALIGN


def pack(dt=1, causal=0, end=0, scale=0.125, cap=0.0, B=2, Lq=16, Lk=16, H=4, Hk=2, D=64, q=None, k=None, v=None, o=None,
         do=None, dq=None, dk=None, dv=None, R=0, strip=0, kv_len=0, prefix=0, q_doc=0, k_doc=0):
    qs, ks = (Lq * H * D, H * D, D), (Lk * Hk * D, Hk * D, D)
    return seq._PACK.pack(dt, causal, end, scale, cap, B, Lq, Lk, H, Hk, D, *(q or qs), *(k or ks), *(v or ks), *(o or qs),
                          *(do or qs), *(dq or qs), *(dk or ks), *(dv or ks), R, strip, kv_len, prefix, q_doc, k_doc)


def test_attention_dimensions_refused(lib):
    ws = lib.seq_attention_workspace_bytes
    assert ws(pack(), 0) >= 0 and ws(pack(), 1) > 0
    for k in ({"dt": 3}, {"B": -1}, {"Lq": -1}, {"Lk": -1}, {"H": 0}, {"Hk": 0}, {"H": 3}, {"D": 0}, {"D": 12}, {"R": -1},
              {"scale": float("inf")}, {"scale": float("nan")}, {"cap": -1.0}, {"cap": float("nan")}, {"q": (-8, 256, 64)}):
        assert ws(pack(**k), 0) == EINVAL, k
    for k in ({"D": 136}, {"Lq": (1 << 20) + 1}, {"Lk": (1 << 20) + 1}, {"R": 1025}, {"B": 1 << 24}, {"H": 1 << 24, "Hk": 1},
              {"B": 1 << 13, "H": 1 << 11}, {"k": (1 << 30, 1 << 23, 64)}, {"B": 1 << 10, "Lq": 1 << 20, "Hk": 1, "H": 64}):
        assert ws(pack(**k), 0) == ERANGE, k
    assert ws(pack(dk=(8, 8, -8)), 0) >= 0 and ws(pack(dk=(8, 8, -8)), 1) == EINVAL    # read by the backward call only


def test_attention_pointers_refused(lib):
    f = lambda a, q=P, k=2 * P, v=3 * P, o=4 * P, lse=5 * P, ws=6 * P, n=1 << 30: lib.seq_attention_forward(
        a, q, k, v, o, lse, ws, n, None)
    for i in range(5):
        args = [P, 2 * P, 3 * P, 4 * P, 5 * P]
        args[i] = None
        assert f(pack(), *args) == EINVAL
    assert f(pack(R=4)) == EINVAL                       # a bias without its strip
    assert f(pack(q_doc=P)) == EINVAL and f(pack(k_doc=P)) == EINVAL
    assert f(pack(), q=P + 8) == EALIGN and f(pack(), lse=5 * P + 2) == EALIGN and f(pack(), ws=6 * P + 4) == EALIGN
    assert f(pack(q=(1024 + 4, 256, 64))) == EALIGN and f(pack(k=(16 * 132, 132, 64))) == EALIGN
    assert f(pack(kv_len=P + 1)) == EALIGN
    assert f(pack(), n=-1) == EWORKSPACE
    assert f(pack(q_doc=P, k_doc=P), ws=None, n=0) == EWORKSPACE
    b = lambda a, *x: lib.seq_attention_backward(a, *x, None)
    good = [P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 7 * P, 8 * P, 9 * P, None, 10 * P, 1 << 30]
    for i in range(9):
        bad = list(good)
        bad[i] = None
        assert b(pack(), *bad) == EINVAL, i


def test_binding_refuses_what_does_not_fit(lib):
    t = torch.zeros
    q, k = t(2, 5, 4, 64), t(2, 7, 2, 64)
    f = pkg.seq_attention_forward
    for args, kw in (((q[0], k, k), {}), ((q, k, k[:, :6]), {}), ((q, k[:1], k[:1]), {}), ((q, k[..., :32], k[..., :32]), {}),
                     ((q, k, k), {"bias": t(3, 9)}), ((q, k, k), {"bias": t(4, 8)}), ((q, k, k), {"bias": t(4, 1)}),
                     ((q, k, k), {"kv_len": t(2)}), ((q, k, k), {"kv_len": t(3, dtype=torch.int32)}),
                     ((q, k, k), {"prefix": t(2, dtype=torch.int32)}), ((q, k, k), {"q_doc": t(2, 5, dtype=torch.int32)}),
                     ((q, k, k), {"q_doc": t(2, 5, dtype=torch.int32), "k_doc": t(2, 5, dtype=torch.int32)}),
                     ((q, k, k), {"out": t(2, 5, 4, 32)}), ((q.transpose(2, 3), k, k), {})):
        with pytest.raises(ValueError):
            f(*args, **kw)
    with pytest.raises(TypeError):
        f(q, k.half(), k.half())
    with pytest.raises(ValueError):
        f(q.double(), k.double(), k.double())
    x, w = t(4, 8), t(8)
    for args in ((x, w[:7], w), (x.t(), w[:4], w[:4]), (t(()), w, w), (t(3, 5, 8)[:, :4], w, w)):
        with pytest.raises(ValueError):
            pkg.seq_layer_norm_forward(*args)
    with pytest.raises(TypeError):
        pkg.seq_layer_norm_forward(x, w.half(), w.half())
    with pytest.raises(TypeError):
        pkg.seq_layer_norm_forward(x.half(), w.half(), w)
    with pytest.raises(ValueError):
        pkg.seq_layer_norm_backward(t(4, 7), x, w, t(4), t(4))
    with pytest.raises(ValueError):
        pkg.seq_rel_bias_forward(t(32), 128)
    with pytest.raises(ValueError):
        pkg.seq_rel_bias_backward(t(4, 8), 32)


def test_grids_of_attention(lib):
    """A launch has less than 2^32 lanes: what would need more is refused
    before anything is enqueued, and only that."""
    ws = lib.seq_attention_workspace_bytes
    many = {"B": 1 << 11, "H": 1 << 10, "Hk": 1 << 10}
    assert ws(pack(**many, Lq=7 * 128), 0) >= 0 and ws(pack(**many, Lq=7 * 128 + 1), 0) == ERANGE
    assert ws(pack(**many, Lq=6 * 64, Lk=64), 1) >= 0 and ws(pack(**many, Lq=6 * 64, Lk=128), 1) == ERANGE
    assert ws(pack(**many, Lq=8 * 64, Lk=1), 1) == ERANGE
    # keys alone make no grid of the forward call
    assert ws(pack(B=1 << 14, H=64, Hk=1, Lq=1, Lk=1 << 17), 0) >= 0
    docs = {"B": 1 << 16, "H": 1, "Hk": 1, "Lq": 1}
    assert ws(pack(**docs, Lk=1 << 15, q_doc=P, k_doc=P), 0) >= 0
    assert ws(pack(**docs, Lk=1 << 16, q_doc=P, k_doc=P), 0) == ERANGE


def test_strides_of_one_are_not_read(lib):
    ws = lib.seq_attention_workspace_bytes
    for far in (1 << 60, (1 << 24) + 8, -8):
        assert ws(pack(Lq=1, q=(256, far, 64), o=(256, far, 64)), 0) >= 0
        assert ws(pack(B=1, k=(far, 128, 64)), 0) >= 0
        assert ws(pack(H=1, Hk=1, v=(1024, 64, far), dk=(1024, 64, far)), 1) >= 0
    assert ws(pack(k=(1 << 40, 128, 64)), 0) >= 0
    assert ws(pack(k=(1 << 45, 128, 64)), 0) == ERANGE
    assert ws(pack(B=1 << 12, k=(1 << 40, 128, 64)), 0) == ERANGE
