"""Tensors that share their memory with another until one of them is written: the cache's calls write their own."""
import pytest
import torch

import paper_2608_20725_amd as pkg

copy_of, lazy = torch._lazy_clone, torch._C._is_cow_tensor
EBUFFER = -8


def pools(device, dt=torch.float32, ct=torch.float32):
    """Keys' and values' pages and scales (or None), all zeros."""
    pages = [torch.zeros((4, 16, 2, 64), dtype=ct, device=device) for _ in range(2)]
    scales = [torch.zeros((4, 16, 2), device=device) for _ in range(2)] if ct != dt else [None, None]
    return pages + scales


def refused(call, *args, **kw):
    """Host memory is refused, behind everything that the binding does."""
    with pytest.raises(pkg.Im2winError) as e:
        call(*args, **kw)
    assert e.value.status == EBUFFER


@pytest.mark.parametrize("ct", [torch.float32, torch.int8])
def test_what_a_call_writes_is_its_own(ct):
    originals = pools("cpu", ct=ct)
    k, v, ks, vs = [None if t is None else copy_of(t) for t in originals]
    x, table = copy_of(torch.ones(2, 3, 2, 64)), copy_of(torch.zeros(2, 4, dtype=torch.int32))
    n, q = copy_of(torch.ones(2, dtype=torch.int32)), copy_of(torch.ones(2, 4, 64))
    freq = pkg.seq_rotary_frequencies(64)
    scales = {} if ks is None else {"k_scale": ks, "v_scale": vs}
    # read
    out, ws = copy_of(torch.zeros(2, 4, 64)), copy_of(torch.zeros(1 << 20, dtype=torch.uint8))
    refused(pkg.seq_paged_attention_forward, q, k, v, table, n, out=out, ws=ws, **scales)
    assert not lazy(out) and not lazy(ws)
    dense = [copy_of(torch.zeros(2, 5, 2, 64)) for _ in range(2)]
    refused(pkg.seq_cache_read, k, v, table, n, 5, k=dense[0], v=dense[1], **scales)
    assert not lazy(dense[0]) and not lazy(dense[1])
    turned = copy_of(torch.zeros(2, 3, 2, 64))
    refused(pkg.seq_rotary_forward, x, freq, out=turned)
    assert not lazy(turned)
    assert all(lazy(t) for t in (k, v, x, table, n, q, *scales.values())), "what is read stays shared"
    # write
    refused(pkg.seq_cache_write, x, x, k, v, table, n, n, **scales)
    assert not lazy(k) and not lazy(v) and not any(lazy(s) for s in scales.values())
    assert lazy(x) and lazy(table) and lazy(n)
    refused(pkg.seq_rotary_backward, x, freq, out=x)
    assert not lazy(x)


@pytest.mark.gpu
@pytest.mark.parametrize("ct", [torch.float32, torch.int8])
def test_the_tensor_copied_from_stays_as_it_was(ct):
    g = torch.Generator().manual_seed(1)
    x = torch.randn((2, 20, 2, 64), generator=g).cuda()
    table = torch.tensor([[0, 3], [2, 1]], dtype=torch.int32, device="cuda")
    n = torch.full((2,), 20, dtype=torch.int32, device="cuda")
    originals, plain = pools("cuda", ct=ct), pools("cuda", ct=ct)
    copies = [None if t is None else copy_of(t) for t in originals]
    results = []
    for k, v, ks, vs in (plain, copies):
        scales = {} if ks is None else {"k_scale": ks, "v_scale": vs}
        pkg.seq_cache_write(x, 2 * x, k, v, table, **scales)
        base = torch.zeros(2, 4, 64, device="cuda")
        out, lse = pkg.seq_paged_attention_forward(x[:, 0].repeat(1, 2, 1), k, v, table, n, out=copy_of(base), **scales)
        dense = torch.zeros(2, 20, 2, 64, device="cuda")
        a, b = pkg.seq_cache_read(k, v, table, n, 20, k=copy_of(dense), v=copy_of(dense), **scales)
        turned = copy_of(a)
        pkg.seq_rotary_forward(turned, pkg.seq_rotary_frequencies(64), out=turned)
        assert not base.any() and not dense.any()
        results.append((out, lse, a, b, turned))
    assert not any(t.any() for t in originals if t is not None)
    assert all(torch.equal(p, c) for p, c in zip(plain, copies) if p is not None)
    assert all(torch.equal(p, c) for p, c in zip(*results))
    assert results[0][0].any() and not torch.equal(results[0][2], results[0][4])
