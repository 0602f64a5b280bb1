"""A cache whose tensors get other storage between calls: append writes where they lie now, attention reads there."""
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch, check_attention
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
def test_calls_follow_the_tensors(e4m3):
    b = Batch(81, [300, 40], hq=8, hkv=2, page=64, e4m3=e4m3)
    cache = b.upload(nsa)
    tensors = [x for x in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale) if x is not None]
    old = [x.detach() for x in tensors]                    # keep the first storage, and see that nothing happens to it
    was = [x.view(torch.uint8).clone() for x in old]
    want = cache.attention(b.dq, b.dtable, b.dlen)
    for x in tensors:
        x.data = x.clone()
    for x in old:
        x.view(torch.uint8).fill_(255)
    got = cache.attention(b.dq, b.dtable, b.dlen)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    cache.append(b.dk, b.dv, b.dtable, b.dlen)
    assert all((x.view(torch.uint8) == 255).all() for x in old)
    assert any(not torch.equal(x.view(torch.uint8), y) for x, y in zip(tensors, was))
    pages, scales = [x.copy() for x in b.pages], [None if x is None else x.copy() for x in b.scales]
    pco.append(b.k, b.v, b.table, b.kv_len, b.cu, pages, scales, b.page)
    o, lse = cache.attention(b.dq, b.dtable, b.dlen)
    check_attention(o, lse, pco.attend(b.q, b.table, b.kv_len, b.cu, pages, scales, b.page))
