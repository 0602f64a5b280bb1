"""The append's factor on the host: what it refuses, before anything is launched."""
import ctypes as C
import inspect

import pytest
import torch

import paper_2508_18224_amd as nsa
from test_paged_cache_pins import P, _shape


def test_the_library_refuses():
    call = lambda f, rot=128: nsa.lib().nsa_sel_cache_append_factor(C.byref(_shape(nsa, n_tokens=3, nseq=3, hq=8, hkv=2)), None, 0, P, 256, P, 256, None, P, P, None, rot, 0, f, P, P, P, P,  # noqa: E731
                                                                    None, None, None)
    for f in (float("nan"), float("inf")):
        assert call(f) == -1
    assert call(1.0) == -1                                  # (channels to turn and no frequencies: nothing here reaches a launch)
    empty = _shape(nsa, n_tokens=0, nseq=0, hq=8, hkv=2)
    for f, rc in ((1.25, 0), (0.0, 0), (-1.0, 0), (float("inf"), -1)):
        assert nsa.lib().nsa_sel_cache_append_factor(C.byref(empty), None, 0, None, 0, None, 0, None, None, None, None, 0, 0, f, None, None, None, None, None, None, None) == rc


def test_the_python_call_refuses():
    cache = nsa.PagedCache(5, 2, page=64, device="cpu")
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    table, kv_len = torch.zeros(3, 4, dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    for factor in (0.0, -1.0, float("nan")):
        with pytest.raises(nsa.NsaSelError, match="factor must be positive"):
            cache.append(k, k, table, kv_len, factor=factor)
    with pytest.raises(TypeError):
        cache.append(k, k, table, kv_len, factor=None)
    for factor in (1, 1.25, torch.tensor(1.1)):
        with pytest.raises(nsa.NsaSelError, match="device tensors"):
            cache.append(k, k, table, kv_len, factor=factor)


def test_the_frequencies_and_their_factor_go_to_both():
    """What rotary_frequencies gives is an argument of each of the calls that it is for."""
    for call in (nsa.rotary, nsa.PagedCache.append):
        assert {"inv_freq", "factor"} <= set(inspect.signature(call).parameters)
