"""Caches and inputs of more than 2^32 bytes: what lies at the far end is what the same call makes at the near end of a small one."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, Batch, check_attention, dev, host
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu
HKV, PAGE = 4, 64


def _far(small, b):
    """A cache with the pages of `small` at its end, 2^32 bytes and more from its beginning, and the table for it."""
    size = small.k_pages.element_size()
    n_pages = 2 ** 32 // (HKV * PAGE * 128 * size) + 5 + b.n_pages
    tensors = []
    for x in (small.k_pages, small.v_pages, small.k_scale, small.v_scale):
        if x is not None:
            y = torch.zeros((n_pages, *x.shape[1:]), dtype=torch.int16 if x.dtype is torch.bfloat16 else torch.uint8 if x.dtype is E4M3 else x.dtype, device="cuda").view(x.dtype)
            y[-b.n_pages:].view(torch.uint8).copy_(x.view(torch.uint8))
            tensors.append(y)
    assert (n_pages - b.n_pages) * HKV * PAGE * 128 * size >= 2 ** 32
    table = torch.where((b.dtable >= 0) & (b.dtable < b.n_pages), b.dtable + (n_pages - b.n_pages), -1)
    return nsa.PagedCache.from_tensors(*tensors), table


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new", [([300, 100, 64, 1], None), ([300, 200, 33], [150, 2, 33]), ([5000], [4500])])
def test_append_and_attention(kv, new, e4m3):
    """In 8 bits scales grow, so that far pages are read and written again."""
    b = Batch(130 + len(kv), kv, new, hq=8, hkv=HKV, page=PAGE, e4m3=e4m3)
    b.k, b.v = b.k * 64, b.v * 64
    near = b.upload(nsa)
    far, table = _far(near, b)
    f = dev(10000.0 ** (-np.arange(0, 128, 2) / 128), torch.float64)
    args = dict(q=b.dq, inv_freq=f, rotated_k=True)
    want = near.append(b.dk, b.dv, b.dtable, b.dlen, b.dcu, **args)
    got = far.append(b.dk, b.dv, table, b.dlen, b.dcu, **args)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for x, y in ((far.k_pages, near.k_pages), (far.v_pages, near.v_pages), (far.k_scale, near.k_scale), (far.v_scale, near.v_scale)):
        if x is not None:
            assert torch.equal(x[-b.n_pages:].view(torch.uint8), y.view(torch.uint8))
            for a in range(0, len(x) - b.n_pages, 4096):   # nothing before them was written
                assert not x[a:min(a + 4096, len(x) - b.n_pages)].view(torch.uint8).any()
    if b.T > 1000:
        return
    idx = dev(b.draw_idx(3, 64), torch.int32)
    for kw in (dict(), dict(idx=idx), dict(window=70)):
        want = near.attention(b.dq, b.dtable, b.dlen, b.dcu, **kw)
        got = far.attention(b.dq, table, b.dlen, b.dcu, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    o, lse = near.attention(b.dq, b.dtable, b.dlen, b.dcu)
    held = [host(near.k_pages), host(near.v_pages)], [None, None] if not e4m3 else [host(near.k_scale), host(near.v_scale)]
    check_attention(o, lse, pco.attend(b.q, b.table, b.kv_len, b.cu, held[0], held[1], PAGE))


@pytest.mark.parametrize("e4m3", [False, True])
def test_tokens_that_lie_far_apart(e4m3):
    """The last token lies more than 2^31 values behind the first."""
    b = Batch(140, [70, 3, 64], [1, 1, 1], hq=8, hkv=HKV, page=PAGE, e4m3=e4m3)
    near, stride = b.upload(nsa), 2 ** 30 + 2 ** 11
    other = Batch(140, [70, 3, 64], [1, 1, 1], hq=8, hkv=HKV, page=PAGE, e4m3=e4m3).upload(nsa)
    whole = torch.empty(2 * stride + 16 * 128, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(whole, (3, 16, 128), (stride, 128, 1))
    rows[:, :8], rows[:, 8:12], rows[:, 12:] = b.dq, b.dk, b.dv
    want = near.append(b.dk, b.dv, b.dtable, b.dlen, b.dcu, q=b.dq, rotated_k=True)
    got = other.append(rows[:, 8:12], rows[:, 12:], b.dtable, b.dlen, b.dcu, q=rows[:, :8], rotated_k=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for x, y in ((other.k_pages, near.k_pages), (other.v_pages, near.v_pages), (other.k_scale, near.k_scale), (other.v_scale, near.v_scale)):
        assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))
