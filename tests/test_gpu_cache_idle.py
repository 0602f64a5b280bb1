"""Idle slots of a padded batch: sequences whose one new token has a negative place.  Nothing is written for them, their rows of the rotated queries and keys are
left as they were, and what those hold does not matter afterwards."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch, check_attention, dev
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n", [9, 300])
def test_idle_slots(n, e4m3):
    lens = np.where(np.arange(n) % 3 == 1, 0, 1 + 7 * (np.arange(n) % 40))
    lens[4] = -3
    idle = lens <= 0
    b = Batch(90 + n, lens, hq=8, hkv=2, page=32, e4m3=e4m3)
    cache = b.upload(nsa)
    freq = 10000.0 ** (-np.arange(0, 128, 2) / 128)
    q_out = torch.full((n, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    k_out = torch.full((n, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    free = torch.from_numpy(~b.live.any(1)).cuda()
    before = [x.view(torch.uint8)[free].clone() for x in (cache.k_pages, cache.v_pages)]
    q, k = cache.append(b.dk, b.dv, b.dtable, b.dlen, q=b.dq, inv_freq=dev(freq, torch.float64), q_out=q_out, k_out=k_out)
    off = torch.from_numpy(idle).cuda()
    assert q[off].isnan().all() and (k[off] == 5.0).all() and not q[~off].isnan().any()
    for x, y in zip((cache.k_pages, cache.v_pages), before):
        assert torch.equal(x.view(torch.uint8)[free], y)
    idx = nsa.select_blocks(torch.rand(n, 2, 5, device="cuda"), None, 4, kv_len=b.dlen)
    assert (idx[off] == -1).all()
    for kw in (dict(idx=idx), dict(window=40), dict()):
        o, lse = cache.attention(q, b.dtable, b.dlen, **kw)
        assert (o[off] == 0).all() and torch.isneginf(lse[off]).all()
        assert torch.isfinite(o[~off].float()).all() and torch.isfinite(lse[~off]).all()
    pages = [x.float().cpu().double().numpy() for x in (cache.k_pages, cache.v_pages)]
    scales = [None if x is None else x.cpu().double().numpy() for x in (cache.k_scale, cache.v_scale)]
    ref = pco.attend(np.nan_to_num(q.float().cpu().double().numpy()), b.table, b.kv_len, None, pages, scales, 32)
    check_attention(o, lse, ref)
