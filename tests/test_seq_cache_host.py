"""Rotary positions and the paged cache on the host: descriptions of the
structs' sizes, refusals of the C interface and of the binding, frequencies,
and the walk through a page table.  No call here reaches a GPU."""
import ctypes
import os
import struct
import subprocess

import pytest
import torch

import paper_2608_20725_amd as pkg
from seq_cache_ref import frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EALIGN, ERANGE, EWORKSPACE, EOVERLAP, EBUFFER = -1, -2, -3, -6, -7, -8
P = 1 << 40  # an aligned address nothing is read from


# seq_rotary_t: dt, interleaved, by_token, amplitude; B, L, H, D, rot; strides of x, y; positions, freq
ROTARY = struct.Struct("@3if11q2P")
# seq_cache_t: dt; B, pages, page, max_pages, Hkv, D; strides of k, v, their scales; table's; k, v, scales, table
CACHE = struct.Struct("@i4x19q5P")
# seq_paged_attention_t: dt, scale, cap; H; strides of q, out; R, strip, len
PAGED = struct.Struct("@i2f4x6q2P")
TRIPLE = struct.Struct("@3q")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.library_path()):
        from paper_2608_20725_amd import build
        build.build()
    lib = ctypes.CDLL(pkg.library_path())
    text, i64, vp, int_ = ctypes.c_char_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.seq_rotary_forward.argtypes = lib.seq_rotary_backward.argtypes = [text, vp, vp, vp]
    lib.seq_cache_write.argtypes = [text, vp, vp, text, text, i64, int_, vp, vp, vp]
    lib.seq_cache_read.argtypes = [text, vp, vp, text, text, i64, int_, vp, vp]
    lib.seq_paged_attention_workspace_bytes.restype = i64
    lib.seq_paged_attention_workspace_bytes.argtypes = [text, i64, int_]
    lib.seq_paged_attention_forward.argtypes = [text, text, vp, vp, vp, vp, i64, vp]
    return lib


def test_descriptions_have_the_structs_layout(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "im2win_seq.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) { printf('
                   '"%zu %zu %zu %zu %zu %zu %zu %zu", sizeof(seq_rotary_t), offsetof(seq_rotary_t, B), '
                   'offsetof(seq_rotary_t, freq), sizeof(seq_cache_t), offsetof(seq_cache_t, table_stride), '
                   'offsetof(seq_cache_t, table), sizeof(seq_paged_attention_t), offsetof(seq_paged_attention_t, len)); '
                   'return 0; }\n')
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    rot, b, freq, cache, stride, table, paged, length = map(
        int, subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split())
    r = ROTARY.pack(0, 0, 0, 0.0, 71, *([0] * 10), 0, 72)
    c = CACHE.pack(0, *([0] * 18), 73, 0, 0, 0, 0, 74)
    a = PAGED.pack(0, 0.0, 0.0, *([0] * 6), 0, 75)
    assert (len(r), len(c), len(a)) == (rot, cache, paged)
    at = lambda s, o: int.from_bytes(s[o:o + 8], "little")
    assert (at(r, b), at(r, freq), at(c, stride), at(c, table), at(a, length)) == (71, 72, 73, 74, 75)


def test_frequencies(lib):
    for rot in (2, 6, 80, 128, 256):
        for opts in ({}, {"base": 5e5}, {"factor": 4.0}, {"factor": 8.0, "trained": 4096.0},
                     {"factor": 32.0, "trained": 8192.0, "low": 1.0, "high": 4.0, "base": 5e5}):
            got = pkg.seq_rotary_frequencies(rot, **opts)
            assert got.shape == (rot // 2,)
            for g, w in zip(got.tolist(), frequencies(rot, **opts)):
                assert abs(g - w) <= 2.0 ** -48 * w  # a few roundings of pow and the line
    for bad in ((1, 1e4), (0, 1e4), (5, 1e4), (4, 0.5), (4, float("nan")), (4, 1e4, 0.5), (4, 1e4, 2.0, -1.0),
                (4, 1e4, 2.0, 100.0, 3.0, 3.0)):
        with pytest.raises(pkg.Im2winError) as e:
            pkg.seq_rotary_frequencies(*bad)
        assert e.value.status == EINVAL
    with pytest.raises(pkg.Im2winError) as e:
        pkg.seq_rotary_frequencies(258)
    assert e.value.status == ERANGE


def rotary(lib, x=P, y=2 * P, dt=1, B=2, L=3, H=4, D=16, rot=16, xs=None, ys=None, pos=0, freq=True, amplitude=1.0, f=0.5,
           backward=False):
    dense = (L * H * D, H * D, D)
    host = (ctypes.c_double * 256)(*([f] * 256))
    a = ROTARY.pack(dt, 0, 0, amplitude, B, L, H, D, rot, *(xs or dense), *(ys or dense), pos,
                               ctypes.addressof(host) if freq else 0)
    return (lib.seq_rotary_backward if backward else lib.seq_rotary_forward)(a, x, y, None)


@pytest.mark.parametrize("backward", [False, True])
def test_rotary_refusals(lib, backward):
    f = lambda **k: rotary(lib, backward=backward, **k)
    for k in ({"x": None}, {"y": None}, {"dt": 3}, {"dt": 16}, {"B": -1}, {"L": -1}, {"H": -1}, {"D": 0}, {"rot": 0},
              {"rot": 3}, {"rot": 18}, {"freq": False}, {"amplitude": float("inf")}, {"amplitude": float("nan")},
              {"f": float("nan")}, {"f": float("inf")}, {"xs": (-1, 64, 16)}, {"ys": (192, 64, -16)}):
        assert f(**k) == EINVAL, k
    for k in ({"D": 258, "rot": 258}, {"D": (1 << 16) + 2}, {"f": 1025.0}, {"f": -1025.0}, {"B": 1 << 31}, {"L": 1 << 31},
              {"H": 1 << 30, "L": 1, "D": 2, "rot": 2}, {"B": 1 << 20, "L": 1 << 20}, {"xs": (1 << 60, 64, 16)},
              {"B": 1, "L": 1 << 30, "D": 64, "rot": 64}, {"B": 1 << 16, "L": 1 << 15, "H": (1 << 31) - 1, "xs": (0, 0, 0)}):
        assert f(**k) == ERANGE, k
    assert f(x=P + 1) == EALIGN and f(y=2 * P + 1) == EALIGN and f(pos=3 * P + 2) == EALIGN
    assert f(dt=0, x=P + 2) == EALIGN
    for k in ({"B": 0}, {"L": 0}, {"H": 0}):
        assert f(x=None, y=None, **k) == 0  # nothing to do, before any device is asked
    assert f() in (EBUFFER, -4)  # buffers that are none, or no device at all


def cache(dt=1, B=2, pages=8, page=16, most=4, Hkv=2, D=64, ks=None, vs=None, kss=(0, 0, 0), vss=(0, 0, 0), ts=None, k=P,
          v=2 * P, k_scale=0, v_scale=0, table=3 * P):
    dense = (page * Hkv * D, Hkv * D, D)
    return CACHE.pack(dt, B, pages, page, most, Hkv, D, *(ks or dense), *(vs or dense), *kss, *vss,
                                 most if ts is None else ts, k or 0, v or 0, k_scale, v_scale, table or 0)


CODED = {"dt": 16, "k_scale": 8 * P, "v_scale": 9 * P, "kss": (32, 2, 1), "vss": (32, 2, 1)}
BAD_CACHE = [
    (EINVAL, [{"dt": 3}, {"dt": 18}, {"B": -1}, {"pages": -1}, {"page": 0}, {"most": -1}, {"Hkv": 0}, {"D": 0}, {"D": 12},
              {"ts": 3}, {"k": 0}, {"v": 0}, {"table": 0}, {"ks": (-8, 128, 64)}, {"vs": (2048, -128, 64)},
              {**CODED, "k_scale": 0}, {**CODED, "v_scale": 0}, {**CODED, "kss": (32, -2, 1)}]),
    (ERANGE, [{"D": 136}, {"page": (1 << 30) + 1}, {"page": 1 << 20, "most": 1025}, {"pages": 1 << 31}, {"B": 1 << 24},
              {"Hkv": 1 << 24}, {"ks": (1 << 60, 128, 64)}, {"ts": 1 << 60}, {**CODED, "vss": (1 << 60, 2, 1)}]),
    (EALIGN, [{"k": P + 8}, {"v": 2 * P + 2}, {"table": 3 * P + 2}, {"ks": (2052, 128, 64)}, {"vs": (2048, 132, 64)},
              {**CODED, "ks": (2052, 128, 64)}, {**CODED, "k_scale": 8 * P + 2}]),
]


def copies(lib, c, k=4 * P, v=5 * P, ks=(8 * 128, 128, 64), vs=(8 * 128, 128, 64), L=8, dt=1, start=6 * P, count=7 * P,
           read=False):
    t = TRIPLE
    ks, vs = (None if s is None else t.pack(*s) for s in (ks, vs))
    if read:
        return lib.seq_cache_read(c, k, v, ks, vs, L, dt, count, None)
    return lib.seq_cache_write(c, k, v, ks, vs, L, dt, start, count, None)


def attends(lib, c, dt=1, scale=0.1, cap=0.0, H=4, qs=(256, 64), os=(256, 64), R=0, strip=0, length=6 * P, q=4 * P,
            out=5 * P, lse=7 * P, ws=None, size=0):
    a = PAGED.pack(dt, scale, cap, H, *qs, *os, R, strip, length or 0)
    return lib.seq_paged_attention_forward(c, a, q, out, lse, ws, size, None)


@pytest.mark.parametrize("status,cases", BAD_CACHE, ids=["einval", "erange", "ealign"])
def test_cache_refusals(lib, status, cases):
    for k in cases:
        c = cache(**k)
        assert copies(lib, c) == status, k
        assert copies(lib, c, read=True) == status, k
        assert attends(lib, c) == status, k
    assert lib.seq_cache_write(None, P, P, None, None, 1, 1, None, None, None) == EINVAL
    assert lib.seq_paged_attention_forward(None, None, P, P, P, None, 0, None) == EINVAL
    assert lib.seq_paged_attention_workspace_bytes(None, 4, 1) == EINVAL


@pytest.mark.parametrize("read", [False, True])
def test_copy_refusals(lib, read):
    f = lambda c=None, **k: copies(lib, c or cache(), read=read, **k)
    for k in ({"k": None}, {"v": None}, {"L": -1}, {"dt": 0}, {"dt": 3}, {"dt": 16}, {"ks": None}, {"vs": None},
              {"ks": (-1, 128, 64)}):
        assert f(**k) == EINVAL, k
    assert f(cache(**CODED), dt=16) == EINVAL
    if read:
        assert f(count=None) == EINVAL
    for k in ({"L": (1 << 30) + 1}, {"L": 1 << 30}, {"ks": (1 << 60, 128, 64)}):
        assert f(**k) == ERANGE, k
    for k in ({"k": 4 * P + 8}, {"v": 5 * P + 2}, {"ks": (1024, 132, 64)}, {"count": 7 * P + 2}):
        assert f(**k) == EALIGN, k
    if not read:
        assert f(start=6 * P + 2) == EALIGN
    assert f(L=0, k=None, v=None, count=None, start=None) == 0
    assert f(cache(B=0, table=0), k=None, v=None, count=None, start=None) == 0


def test_paged_attention_refusals(lib):
    f = lambda c=None, **k: attends(lib, c or cache(), **k)
    for k in ({"q": None}, {"out": None}, {"lse": None}, {"length": 0}, {"dt": 0}, {"dt": 16}, {"H": 0}, {"H": 3},
              {"scale": float("nan")}, {"cap": -1.0}, {"cap": float("inf")}, {"R": -1}, {"R": 4}, {"qs": (-1, 64)}):
        assert f(**k) == EINVAL, k
    for k in ({"H": 1 << 24}, {"R": 1025, "strip": P}, {"qs": (1 << 60, 64)}):
        assert f(**k) == ERANGE, k
    for k in ({"q": 4 * P + 8}, {"out": 5 * P + 2}, {"lse": 7 * P + 2}, {"length": 6 * P + 1}, {"qs": (260, 64)},
              {"os": (256, 68)}, {"R": 4, "strip": P + 2}, {"ws": P + 8}):
        assert f(**k) == EALIGN, k
    assert f(size=-1) == EWORKSPACE
    assert f(cache(B=0, table=0), q=None, out=None, lse=None, length=0) == 0
    ws = lib.seq_paged_attention_workspace_bytes
    assert ws(cache(), 3, 1) == EINVAL and ws(cache(), 4, 0) == EINVAL and ws(cache(), 1 << 24, 1) == ERANGE
    assert ws(cache(most=0), 4, 1) == 0                      # no keys to split
    assert ws(cache(most=8), 4, 1) == 0                      # 128 keys: a few steps
    assert ws(cache(most=4096), 4, 1) >= 2 * 2 * 4 * 68 * 4  # split: 4 rows of 64 sums each


def test_binding_refusals(lib):
    k = torch.zeros(2, 3, 2, 64)
    pages, table, length = torch.zeros(4, 16, 2, 64), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    codes, scale = torch.zeros(4, 16, 2, 64, dtype=torch.int8), torch.zeros(4, 16, 2)
    freq = torch.zeros(32, dtype=torch.float64)
    for fn in (pkg.seq_rotary_forward, pkg.seq_rotary_backward):
        for bad in ((k, freq.float()), (k, freq[None]), (k, freq[::2]), (k[0], freq), (k.transpose(2, 3), freq),
                    (k, freq, length.long()), (k, freq, length[:1]), (k, freq, torch.zeros(2, 4, dtype=torch.int32))):
            with pytest.raises(ValueError):
                fn(*bad)
        with pytest.raises(ValueError):
            fn(k, freq, out=k.half())
    w = pkg.seq_cache_write
    for bad in ((k, k, pages, pages[:3], table), (k, k, pages, pages.half(), table), (k, k, pages, pages, table.long()),
                (k, k, pages, pages, table[0]), (k, k, pages, pages, table.t()), (k, k[:1], pages, pages, table),
                (k[:, :, :1], k[:, :, :1], pages, pages, table), (k, k, pages, pages, table, length[:1]),
                (k, k, pages, pages, table, None, length.long()), (k, k, pages, pages, table, None, None, scale, scale),
                (k, k, codes, codes, table), (k, k, codes, codes, table, None, None, scale, scale[:3]),
                (k, k, codes, codes, table, None, None, scale, scale.double()), (k, k, pages[0], pages[0], table)):
        with pytest.raises(ValueError):
            w(*bad)
    with pytest.raises(TypeError):
        w(k.half(), k.half(), pages, pages, table)
    with pytest.raises(TypeError):
        w(k, k.half(), codes, codes, table, None, None, scale, scale)
    with pytest.raises(TypeError):
        pkg.seq_cache_read(pages, pages, table, length, 8, dtype=torch.float16)
    with pytest.raises(ValueError):
        pkg.seq_cache_read(pages, pages, table, length, 8, k=k)
    a = pkg.seq_paged_attention_forward
    q = torch.zeros(2, 4, 64)
    for bad in ((k, pages, pages, table, length), (q[:1], pages, pages, table, length), (q[..., :32], pages, pages, table, length),
                (q, pages, pages, table, length.long()), (q, pages, pages, table, length[:1])):
        with pytest.raises(ValueError):
            a(*bad)
    for bad in (torch.zeros(4, 8), torch.zeros(3, 9), torch.zeros(4, 1), torch.zeros(4, 9).double()):
        with pytest.raises(ValueError):
            a(q, pages, pages, table, length, bias=bad)
    with pytest.raises(TypeError):
        a(q.half(), pages, pages, table, length)
    for bad in ((None, pages, pages, table, length), (q, pages, pages, table, 3)):
        with pytest.raises(TypeError):
            a(*bad)
    for bad in ((q, pages, pages, table, None), (q.double(), pages, pages, table, length)):
        with pytest.raises(ValueError):
            a(*bad)
    with pytest.raises(TypeError):
        pkg.seq_cache_read(pages, pages, table, length, 2.5)
    with pytest.raises(ValueError):
        pkg.seq_cache_read(pages, pages, table, length, -1)
    for ws in (torch.zeros(1).expand(1 << 20), torch.zeros(1 << 10)[::2]):
        with pytest.raises(ValueError):
            a(q, pages, pages, table, length, ws=ws)
    # host memory is refused by its address
    for call in (lambda: a(q, pages, pages, table, length), lambda: w(k, k, pages, pages.clone(), table),
                 lambda: pkg.seq_cache_read(pages, pages, table, length, 8), lambda: pkg.seq_rotary_forward(k, freq)):
        with pytest.raises(pkg.Im2winError) as e:
            call()
        assert e.value.status in (EBUFFER, -4) and "seq_" in str(e.value)


def test_walk_through_a_table(tmp_path):
    """page_of and held_tokens, as the kernels use them, over good and bad
    entries and positions."""
    src = tmp_path / "w.cpp"
    src.write_text('#include "seq_pages.hpp"\n#include <cstdio>\nusing namespace im2win;\nint main() {\n'
                   'const int32_t row[6] = {3, -1, 7, 8, -2147483647 - 1, 2147483647};\n'
                   'for (int64_t i = -2; i < 8; ++i) printf("%d ", page_of(row, i, 6, 8));\n'
                   'for (int64_t i = 0; i < 6; ++i) printf("%d ", page_of(row, i, 6, 0));\n'
                   'printf("%d ", page_of(nullptr, 0, 0, 8));\n'
                   'const int32_t n[6] = {-2147483647 - 1, -1, 0, 95, 96, 2147483647};\n'
                   'for (int32_t v : n) printf("%d ", held_tokens(v, 6, 16));\n'
                   'printf("%d %d", held_tokens(2147483647, 1 << 20, 1 << 10), held_tokens(5, 0, 16));\nreturn 0; }\n')
    exe = str(tmp_path / "w")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_20725_amd", "csrc"),
                    str(src), "-o", exe], check=True)
    got = list(map(int, subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()))
    assert got == [-1, -1, 3, -1, 7, -1, -1, -1, -1, -1] + [-1] * 6 + [-1] + [0, 0, 0, 95, 96, 96] + [1 << 30, 0]
