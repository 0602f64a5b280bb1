"""The factor of stretched frequencies in the append, as the rotation of the training path has it."""
import functools

import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch, dev
from oracle import paged_cache_oracle as pco
from test_gpu_cache_append import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [[70, 1, 33], [4000, 300, 2]])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True), (32, False)])
def test_same_bits_as_the_rotation(rot, interleaved, tokens):
    """Queries, keys and what lies in the pages, few tokens and many."""
    T = sum(tokens)
    cu = dev(np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32), torch.int32)
    q, k = (torch.randn(T, h, 128, device="cuda").to(torch.bfloat16) for h in (8, 2))
    f, factor = nsa.rotary_frequencies(rot, scaling="parts", stretch=4.0)
    assert factor > 1.1
    per = -(-max(tokens) // 64)
    table = torch.arange(3 * per, dtype=torch.int32, device="cuda").view(3, per)
    x, y = nsa.rotary(q, k, f, cu, interleaved=interleaved, factor=factor)
    for dtype in (torch.bfloat16, torch.float8_e4m3fn):
        cache = nsa.PagedCache(3 * per, 2, page=64, dtype=dtype)
        a, b = cache.append(k, k, table, cu.diff(), cu, q=q, inv_freq=f, interleaved=interleaved, factor=factor, rotated_k=True)
        assert torch.equal(a, x) and torch.equal(b, y)
        if dtype is torch.bfloat16:
            keys, values = cache.read(table, cu.diff(), cu, tokens=T)
            assert torch.equal(keys, y) and torch.equal(values, k)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new,hq,hkv,page,rot,interleaved", [
    ([1000, 64, 65, 63, 1], None, 8, 2, 64, 128, False), ([300, 129, 128], None, 28, 4, 128, 64, True), ([90, 7, 300], [60, 7, 31], 8, 2, 16, 96, False),
    ([4200], [4100], 4, 2, 64, 128, False), ([700, 800], [650, 800], 2, 1, 256, 32, True)])
def test_against_64_bits(kv, new, hq, hkv, page, rot, interleaved, e4m3, monkeypatch):
    """The append's own test with a rotation that multiplies the channels that turn: pages, scales that grow, rows that leave, whatever form the launch takes.  (1.25 is exact in all formats, so its
    bounds hold: they are 2^4 times what a sum of two products and a factor lose.)"""
    factor, plain = 1.25, pco.rotate

    def rotate(x, place, inv_freq, interleaved=False):
        y = plain(x, place, inv_freq, interleaved)
        y[..., :2 * len(inv_freq)] *= factor
        return y

    monkeypatch.setattr(pco, "rotate", rotate)
    monkeypatch.setattr(nsa.PagedCache, "append", functools.partialmethod(nsa.PagedCache.append, factor=factor))
    _run(Batch(401 + rot, kv, new, hq=hq, hkv=hkv, page=page, e4m3=e4m3), rot, interleaved)


def test_a_prompt_and_its_training_step_agree():
    """With part of the head turned the scale of the softmax cannot make up for a missing factor: what the training path's attention gives, the cache gives too."""
    T, hq, hkv = 200, 8, 2
    q, k, v = (torch.randn(T, h, 128, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    f, factor = nsa.rotary_frequencies(64, scaling="parts", stretch=8.0)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    a, b = nsa.rotary(q, k, f, factor=factor)
    idx = nsa.window_blocks(T, hkv, 512, cu)
    o, lse = nsa.SelAttention(T, hq, hkv, idx.shape[2], bwd=False).forward(a, b, v, idx, cu)
    cache = nsa.PagedCache(4, hkv, page=64)
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    r, _ = cache.append(k, v, table, cu[1:], cu, q=q, inv_freq=f, factor=factor)
    o2, lse2 = cache.attention_chunk(r, table, cu[1:], cu)
    size = float(a.float().norm(dim=-1).max() * b.float().norm(dim=-1).max()) * 128 ** -0.5          # of a score's products, at most
    assert float((lse - lse2).abs().max()) <= 2 * (2.0 ** -17 * size + 2.0 ** -21 * float(lse.abs().max()) + 2.0 ** -20)
