"""Pieces of prompts over a cached prefix: hundreds of new tokens of a sequence, whose own keys are in the cache with the earlier ones; sequences that share a prefix's pages."""
import numpy as np
import pytest

from cache_util import Batch
from test_gpu_cache_attention import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new,hq,hkv,page", [([1700], [700], 28, 4, 64), ([900, 2300, 40], [513, 300, 40], 16, 2, 128), ([1000, 77], [259, 77], 24, 8, 32)])
def test_pieces_of_prompts(kv, new, hq, hkv, page, e4m3):
    b = Batch(150 + hq, kv, new, hq=hq, hkv=hkv, page=page, e4m3=e4m3, pad=2, before=1)
    _run(b)
    _run(b, window=333)
    _run(b, b.draw_idx(8, 64), gate=True, acc=True)


def test_sequences_that_share_a_prefix():
    """Their tables name the same pages up to where they part."""
    b = Batch(160, [640, 700, 650], [100, 160, 110], hq=8, hkv=2, page=64)
    shared = 8                                             # pages of the first 512 tokens
    b.table[1:, :shared] = b.table[0, :shared]
    assert len(np.unique(b.table[:, :shared])) == shared
    _run(b)
    _run(b, b.draw_idx(6, 64))
