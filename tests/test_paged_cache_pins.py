"""The oracle of the paged cache, pinned to the oracles of the training path, to closed forms and to torch's own conversions; and what the
calls refuse, without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from cache_util import Batch
from oracle import nsa_sel_oracle as orc
from oracle import paged_cache_oracle as pco
from oracle import topk_select_oracle as tko


def test_attention_over_pages_is_attention_over_tokens():
    """Pages filled by append; every token is a new one, so the training path's forward is the answer."""
    L, hq, hkv, page = 150, 4, 2, 16
    b = Batch(1, [L], [L], hq=hq, hkv=hkv, page=page)
    pages = [np.full_like(x, np.nan) for x in b.pages]
    pco.append(b.k, b.v, b.table, b.kv_len, b.cu, pages, [None, None], page)
    idx = b.draw_idx(3, 64)
    cu = np.array([0, L], dtype=np.int32)
    for window in (0, 40):
        got = pco.attend(b.q, b.table, b.kv_len, b.cu, pages, [None, None], page, idx=idx, window=window)
        ref = orc.forward(b.q, b.k, b.v, idx, cu, window=window)
        assert np.allclose(got[0], ref[0], atol=1e-12) and np.allclose(got[1], ref[1], atol=1e-12)
    every = np.tile(np.arange(3, dtype=np.int32), (L, hkv, 1))
    ref = orc.forward(b.q, b.k, b.v, every, cu)
    got = pco.attend(b.q, b.table, b.kv_len, b.cu, pages, [None, None], page)
    assert np.allclose(got[0], ref[0], atol=1e-12) and np.allclose(got[1], ref[1], atol=1e-12)


def test_rounding_is_torchs():
    x = np.concatenate([np.random.default_rng(2).standard_normal(20000) * s for s in (1e-3, 1.0, 100.0)])
    x = np.concatenate([x, np.arange(-40, 41) / 2.0 ** 11, [448.0, -448.0, 0.0]])
    x = np.clip(x, -448, 448).astype(np.float32).astype(np.float64)
    t = torch.from_numpy(x).to(torch.float32)
    assert np.array_equal(pco.to_e4m3(x), t.to(torch.float8_e4m3fn).to(torch.float64).numpy())
    assert np.array_equal(pco.to_bf16(x), t.to(torch.bfloat16).to(torch.float64).numpy())
    assert np.isnan(pco.to_e4m3(np.array([np.inf, -np.inf, np.nan]))).all() and pco.to_e4m3(np.array([1e9]))[0] == 448.0


def test_scale_is_the_least_power_of_two():
    for a in (1e-30, 1.0, 447.9, 448.0, 448.1, 3e38):
        s = pco.least_scale(np.array([a, -a / 3, np.nan, np.inf]))
        assert np.log2(s) == int(np.log2(s)) and (a <= 448 * s or s == 2.0 ** 119) and (a > 224 * s or s == 2.0 ** -100)


def test_rotation_is_a_rotation_by_the_place():
    x = np.random.default_rng(3).standard_normal((3, 128))
    f = 10000.0 ** (-np.arange(0, 64, 2) / 64)
    for il in (False, True):
        y = pco.rotate(x, 12345, f, il)
        assert np.allclose((y * y).sum(1), (x * x).sum(1)) and np.array_equal(y[:, 64:], x[:, 64:])
        # scores depend on the distance of places alone
        a = (pco.rotate(x, 700, f, il) * pco.rotate(x[::-1], 650, f, il)).sum(1)
        c = (pco.rotate(x, 50, f, il) * x[::-1]).sum(1)
        assert np.allclose(a, c)
    assert np.array_equal(pco.rotate(x, 0, f, False), x)


@pytest.mark.parametrize("block", [64, 128])
def test_selection_is_that_of_a_sequence(block):
    """The last tokens of sequences, as rows of a batch in which all tokens are there."""
    lens, new = [300, 5, 129], [4, 5, 1]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    x = np.round(np.random.default_rng(4).standard_normal((sum(lens), 2, 8)), 1).astype(np.float32)
    ref = tko.select_blocks(x, cu, 4, block=block)
    rows = np.concatenate([np.arange(cu[s + 1] - n, cu[s + 1]) for s, n in enumerate(new)])
    got = pco.select(x[rows], np.array(lens), np.concatenate([[0], np.cumsum(new)]), 4, block=block)
    assert np.array_equal(got, ref[rows])


# ---- what is refused, on the host ------------------------------------------------------------------------------------------
P = C.c_void_p(4096)
ODD = C.c_void_p(4104)


def _shape(nsa, **kw):
    from paper_2508_18224_amd.binding import CacheShape
    d = dict(n_tokens=4, nseq=4, hq=8, hkv=2, d=128, dtype=1, page=64, n_pages=10, max_pages=30, block=64, topk=16, window=0, scale=0.0)
    d.update(kw)
    return CacheShape(*[d[n] for n, _ in CacheShape._fields_])


def _append(L, s, **kw):
    a = dict(Q=P, qs=1024, K=P, ks=256, V=P, vs=256, cu=None, kv_len=P, table=P, inv=P, rot=128, il=0, kp=P, vp=P, kscale=P, vscale=P,
             qo=P, ko=None)
    a.update(kw)
    return L.nsa_sel_cache_append(C.byref(s), *a.values(), None)


def _attend(L, s, **kw):
    a = dict(Q=P, idx=P, cu=None, kv_len=P, table=P, kp=P, vp=P, kscale=P, vscale=P, gate=None, acc=None, O=C.c_void_p(8192), LSE=P, ws=P,
             n=1 << 40)
    a.update(kw)
    return L.nsa_sel_cache_attention(C.byref(s), *a.values(), None)


def test_shapes_refused():
    import paper_2508_18224_amd as nsa
    L = nsa.lib()
    n = C.c_size_t()
    assert L.nsa_sel_cache_workspace_bytes(C.byref(_shape(nsa)), C.byref(n)) == 0 and n.value > 0
    assert L.nsa_sel_cache_workspace_bytes(None, C.byref(n)) == -1
    for kw, rc in ((dict(hq=9), -1), (dict(hq=18), -1), (dict(nseq=-1), -1), (dict(n_tokens=-1), -1), (dict(nseq=0), -1), (dict(dtype=2), -1),
                   (dict(n_pages=-1), -1), (dict(max_pages=-1), -1), (dict(window=-1), -1), (dict(d=64), -2), (dict(page=48), -2),
                   (dict(page=8), -2), (dict(page=512), -2), (dict(block=32), -2), (dict(topk=33), -2), (dict(topk=-1), -2),
                   (dict(max_pages=1 << 25), -2), (dict(n_tokens=1 << 29, nseq=1), -2)):
        assert L.nsa_sel_cache_workspace_bytes(C.byref(_shape(nsa, **kw)), C.byref(n)) == rc, kw
        assert _attend(L, _shape(nsa, **kw)) == rc, kw
    assert L.nsa_sel_cache_workspace_bytes(C.byref(_shape(nsa, topk=0, block=0)), C.byref(n)) == 0


def test_pointers_refused():
    import paper_2508_18224_amd as nsa
    L = nsa.lib()
    s = _shape(nsa)
    for kw in (dict(K=None), dict(V=None), dict(K=ODD), dict(V=ODD), dict(Q=ODD), dict(qo=ODD), dict(ko=ODD), dict(kv_len=None), dict(table=None),
               dict(kp=None), dict(vp=ODD), dict(kscale=None), dict(vscale=None), dict(qo=None), dict(Q=None), dict(inv=None), dict(rot=24),
               dict(rot=144), dict(rot=-16), dict(ks=248), dict(vs=260), dict(qs=1020), dict(qs=8), dict(inv=C.c_void_p(4100)),
               dict(Q=P, qo=P, qs=2048), dict(ko=P, K=P, ks=512)):
        assert _append(L, s, **kw) == -1, kw
    assert _append(L, _shape(nsa, nseq=2)) == -1                              # no cu_seqlens and another number of tokens
    assert _append(L, _shape(nsa, n_tokens=0, nseq=0), K=None, V=None) == 0   # nothing to do
    for kw in (dict(Q=None), dict(Q=ODD), dict(idx=None), dict(idx=C.c_void_p(4098)), dict(kv_len=None), dict(table=None), dict(kp=ODD),
               dict(vscale=None), dict(O=None), dict(O=P), dict(LSE=None), dict(acc=P), dict(gate=P, acc=ODD), dict(gate=C.c_void_p(4098)),
               dict(ws=None), dict(ws=ODD)):
        assert _attend(L, s, **kw) == -1, kw
    assert _attend(L, _shape(nsa, topk=0)) == -1                              # idx without columns
    need = C.c_size_t()
    L.nsa_sel_cache_workspace_bytes(C.byref(s), C.byref(need))
    assert _attend(L, s, n=need.value - 1) == -3
    sel = L.nsa_sel_select_blocks_cached
    for args, rc in (((P, 8, None, None, 1, 2, P), -1), ((P, 8, None, P, 1, 2, None), -1), ((P, 8, None, P, -1, 2, P), -1),
                     ((P, 0, None, P, 1, 2, P), -2), ((P, 16385, None, P, 1, 2, P), -2), ((C.c_void_p(4097), 8, None, P, 1, 2, P), -1)):
        assert sel(C.byref(s), *args, None) == rc, args
    assert sel(None, P, 8, None, P, 1, 2, P, None) == -1
    assert sel(C.byref(_shape(nsa, nseq=2)), P, 8, None, P, 1, 2, P, None) == -1
    for kw, rc in ((dict(block=32), -2), (dict(topk=0), -2), (dict(topk=33), -2), (dict(nseq=0), -1)):
        assert sel(C.byref(_shape(nsa, **kw)), P, 8, None, P, 1, 2, P, None) == rc, kw


def test_binding_refuses_wrong_tensors():
    """Types, shapes, devices and layouts, before the library sees an address."""
    import paper_2508_18224_amd as nsa
    E = nsa.NsaSelError
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    z = torch.zeros
    good = z(5, 2, 64, 128, dtype=bf)
    for args in ((good.float(), good), (good, good[:4]), (good, good, z(5, 2), z(5, 2)), (good[..., :64], good[..., :64]), (good.to(f8), good.to(f8)),
                 (good.to(f8), good.to(f8), z(5, 2), z(5, 1)), (good.to(f8), good, z(5, 2), z(5, 2)), (z(5, 2, 48, 128, dtype=bf), z(5, 2, 48, 128, dtype=bf)),
                 (good.transpose(1, 2), good.transpose(1, 2)), (None, None)):
        with pytest.raises(E):
            nsa.PagedCache.from_tensors(*args)
    with pytest.raises(E):
        nsa.PagedCache(5, 2, dtype=torch.float16, device="cpu")
    with pytest.raises(E):
        nsa.PagedCache(5, 2, page=24, device="cpu")
    assert nsa.PagedCache(5, 2, dtype=f8, device="cpu").k_scale.shape == (5, 2)
    cache = nsa.PagedCache(5, 2, device="cpu")
    i32 = torch.int32
    k, q, table, kv_len = z(3, 2, 128, dtype=bf), z(3, 8, 128, dtype=bf), z(3, 4, dtype=i32), z(3, dtype=i32)
    ok = dict(k=k, v=k, table=table, kv_len=kv_len)
    bad = [dict(k=k.float()), dict(k=k[:, :1]), dict(v=k[:2]), dict(k=k[..., ::2]), dict(table=table.long()), dict(table=table[0]), dict(kv_len=kv_len.long()),
           dict(kv_len=kv_len[:2]), dict(cu=z(3, dtype=i32)), dict(cu=z(4)), dict(table=table[:2], kv_len=kv_len[:2]), dict(q=q.float()),
           dict(q=q[:2]), dict(q_out=q), dict(q=q, q_out=q.float()), dict(k_out=q), dict(inv_freq=z(64)), dict(table=table.t().contiguous().t()),
           dict(k=z(3, 2, 129, dtype=bf)[..., 1:]), dict(k=z(3, 260, dtype=bf)[:, 4:].view(3, 2, 128)),
           dict(k=torch.as_strided(z(1000, dtype=bf), (3, 2, 128), (128, 128, 1)))]
    for kw in bad:
        with pytest.raises(E):
            cache.append(**{**ok, **kw})
    with pytest.raises(E):                                                   # everything fits, but there is no GPU here
        cache.append(**ok, q=q, inv_freq=z(64, dtype=torch.float64))
    ok = dict(q=q, table=table, kv_len=kv_len)
    idx, gate = z(3, 2, 4, dtype=i32), z(3, 8)
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(q=z(3, 8, 256, dtype=bf)[..., ::2]), dict(idx=idx.long()), dict(idx=idx[:2]), dict(idx=idx[..., :0]),
               dict(gate=gate.double()), dict(o_acc=q), dict(gate=gate, o_acc=q.float()), dict(out=q.float()), dict(lse=gate.double()),
               dict(cu=z(3, dtype=i32)), dict(ws=z(4)), dict(window=-1), dict(window=2 ** 32 + 5), dict(idx=idx, block=2 ** 32 + 64), dict(idx=idx, block=32), dict(idx=z(3, 2, 40, dtype=i32))):
        with pytest.raises(E):
            cache.attention(**{**ok, **kw})
    x = z(3, 2, 8)
    for args, kw in (((x, None, 4), dict(kv_len=kv_len[:2])), ((x, None, 4), dict(kv_len=kv_len.long())), ((x, None, 4), dict(kv_len=kv_len, causal=False)),
                     ((x, z(3, dtype=i32), 4), dict(kv_len=kv_len)), ((x.double(), None, 4), dict(kv_len=kv_len))):
        with pytest.raises(E):
            nsa.select_blocks(*args, **kw)
