"""Lengths far below zero with several new tokens of a sequence, and windows of any size beside them: nothing is seen, and the other sequences are as they were."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch
from chunk_util import attend_chunks, check_chunks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [0, 1, 5, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 1])
@pytest.mark.parametrize("length", [-2 ** 31, -2 ** 30 - 1, -2 ** 30, -1, 0])
def test_several_tokens(length, window):
    b = Batch(176, [70, 300, 40], [20, 130, 7], hq=8, hkv=2, page=32)
    cache = b.upload(nsa)
    keys, _ = cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T)
    b.kv_len[0] = b.kv_len[2] = length
    b.dlen[0] = b.dlen[2] = length
    o, lse = cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, window=window)
    k, v = cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T)
    for at in (slice(0, 20), slice(150, 157)):
        assert (o[at] == 0).all() and torch.isneginf(lse[at]).all() and (k[at] == 0).all() and (v[at] == 0).all()
    assert torch.equal(k[20:150], keys[20:150])
    check_chunks(o, lse, attend_chunks(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, 32, window=window), keys=300, most=np.nanmax(np.abs(b.pages[1])))
