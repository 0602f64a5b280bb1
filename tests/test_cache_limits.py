"""Calls over a paged cache that no launch can hold (2^32 work-items) are refused before any launch, the workspace's size with them; on the host.
Only refused calls are made, and sizes asked for: no address here is one of memory."""
import ctypes as C

import pytest

import paper_2508_18224_amd as nsa
from paper_2508_18224_amd.binding import Shape
from test_paged_cache_pins import P, _append, _attend, _shape

OK, UNSUPPORTED = 0, -2


def _need(s):
    n = C.c_size_t(77)
    return nsa.lib().nsa_sel_cache_workspace_bytes(C.byref(s), C.byref(n)), n.value


@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_of_selected_blocks(dtype):
    """A row a workgroup of 256."""
    for hkv, g in ((1, 8), (8, 1), (4, 3), (1 << 20, 1)):
        T = -(-(1 << 24) // hkv)
        for nseq in (1, T):
            assert _need(_shape(nsa, n_tokens=T - 1, nseq=min(nseq, T - 1), hq=hkv * g, hkv=hkv, dtype=dtype))[0] == OK
            s = _shape(nsa, n_tokens=T, nseq=nseq, hq=hkv * g, hkv=hkv, dtype=dtype)
            assert _need(s)[0] == UNSUPPORTED
            assert _attend(nsa.lib(), s, cu=P) == UNSUPPORTED


def test_every_key_without_a_join_where_there_are_too_many_rows_for_it():
    """Whole rows then, which need no workspace: the launch that joins parts has a workgroup for every token and head."""
    kw = dict(hq=64, hkv=8, topk=0, max_pages=4096)
    assert _need(_shape(nsa, n_tokens=(1 << 18) - 1, nseq=1, **kw))[1] > 0
    for T in (1 << 18, 1 << 20, (1 << 22) - 16):
        assert _need(_shape(nsa, n_tokens=T, nseq=1, **kw)) == (OK, 0)
    s = _shape(nsa, n_tokens=1 << 22, nseq=1, **kw)      # two tokens of eight heads a workgroup
    assert _need(s)[0] == UNSUPPORTED and _attend(nsa.lib(), s, idx=None, cu=P) == UNSUPPORTED


def test_append():
    L = nsa.lib()
    for dtype, T, nseq, page in ((0, 1 << 24, 1, 64), (0, 1 << 26, 1 << 20, 256), (1, 1 << 27, 1 << 20, 16), (1, 1 << 27, 1, 256)):
        s = _shape(nsa, n_tokens=T, nseq=nseq, hq=8, hkv=8, dtype=dtype, page=page)
        assert _append(L, s, qs=1024, ks=1024, vs=1024, cu=P, ko=C.c_void_p(8192)) == UNSUPPORTED
    s = _shape(nsa, n_tokens=1 << 24, nseq=1 << 24, hq=8, hkv=1, dtype=1)   # single tokens: a workgroup for K and one for V
    assert _append(L, s, qs=1024, ks=1024, vs=1024) == UNSUPPORTED


def test_selection():
    """Four rows a workgroup of 256; of a large training batch 32."""
    L = nsa.lib()
    s = _shape(nsa, n_tokens=1 << 26, nseq=1, hq=1, hkv=1, topk=8)
    assert L.nsa_sel_select_blocks_cached(C.byref(s), P, 8, P, P, 1, 2, P, None) == UNSUPPORTED
    t = Shape(1 << 29, 1, 1, 1, 128, 64, 1, 1, 0.0, 0)
    assert L.nsa_sel_select_blocks(C.byref(t), P, 8, P, 1, 2, P, None) == UNSUPPORTED
