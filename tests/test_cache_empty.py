"""Batches without a new token: nothing to do, whatever the addresses."""
import ctypes as C

import pytest
import torch

import paper_2508_18224_amd as nsa
from paper_2508_18224_amd.binding import Shape
from test_paged_cache_pins import _shape


def test_the_library_has_nothing_to_select():
    L = nsa.lib()
    for kw in (dict(nseq=0), dict(nseq=3)):
        s = _shape(nsa, n_tokens=0, **kw)
        assert L.nsa_sel_select_blocks_cached(C.byref(s), None, 8, None, None, 1, 2, None, None) == 0
        assert L.nsa_sel_select_blocks_cached(C.byref(s), None, 8, None, None, -1, 2, None, None) == -1
    assert L.nsa_sel_select_blocks_cached(C.byref(_shape(nsa, n_tokens=0, nseq=0, topk=33)), None, 8, None, None, 1, 2, None, None) == -2
    assert L.nsa_sel_select_blocks(C.byref(Shape(0, 1, 8, 2, 128, 64, 4, 1, 0.0, 0)), None, 8, None, 1, 2, None, None) == 0


@pytest.mark.gpu
def test_selection_of_an_empty_batch():
    """As append and attention have it: no sequences, and sequences without new tokens; the same call with tokens besides."""
    x, kv_len = torch.rand(3, 2, 8, device="cuda"), torch.tensor([5, 300, 64], dtype=torch.int32, device="cuda")
    starts = torch.zeros(4, dtype=torch.int32, device="cuda")
    for out in (None, torch.empty(0, 2, 4, dtype=torch.int32, device="cuda")):
        assert nsa.select_blocks(x[:0], None, 4, kv_len=kv_len[:0], out=out).shape == (0, 2, 4)
        assert nsa.select_blocks(x[:0], starts, 4, kv_len=kv_len, out=out).shape == (0, 2, 4)
        assert nsa.select_blocks(x[:0], starts[:2], 4, out=out).shape == (0, 2, 4)
    torch.cuda.synchronize()
    assert nsa.select_blocks(x, None, 4, kv_len=kv_len).shape == (3, 2, 4)
