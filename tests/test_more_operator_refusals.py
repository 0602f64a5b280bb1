"""What the rotation, the read and the attention of pieces refuse, on the host: nothing here reaches a launch."""
import ctypes as C

import pytest
import torch

import paper_2508_18224_amd as nsa
from paper_2508_18224_amd.binding import RotaryShape
from test_paged_cache_pins import P, _shape

OK, EINVAL, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
ODD = C.c_void_p(4098)
Q2 = C.c_void_p(8192)
BF, I32 = torch.bfloat16, torch.int32


# ---- the C ABI ---------------------------------------------------------------------------------------------------------------
def _rotary(s, q=P, qs=1024, k=P, ks=256, cu=P, pos=None, f=P, qo=Q2, qos=1024, ko=Q2, kos=256):
    return nsa.lib().nsa_sel_rotary(C.byref(s), q, qs, k, ks, cu, pos, f, qo, qos, ko, kos, None)


def _rs(**kw):
    v = dict(n_tokens=5, nseq=2, hq=8, hkv=2, d=128, rot=128, interleaved=0, inverse=0, factor=1.0)
    v.update(kw)
    return RotaryShape(*(v[n] for n, _ in RotaryShape._fields_))


def test_rotary_refuses():
    for kw in (dict(n_tokens=-1), dict(nseq=-1), dict(nseq=0), dict(hq=0), dict(hkv=-1), dict(rot=8), dict(rot=144), dict(rot=-16), dict(factor=float("nan")),
               dict(factor=float("inf"))):
        assert _rotary(_rs(**kw)) == EINVAL, kw
    for kw in (dict(d=64), dict(hq=65536), dict(hq=1, hkv=65536), dict(n_tokens=2 ** 31 - 1, hq=64)):
        assert _rotary(_rs(**kw), qs=1 << 24, ks=1 << 24, qos=1 << 24, kos=1 << 24) == UNSUPPORTED, kw
    assert nsa.lib().nsa_sel_rotary(None, P, 1024, P, 256, P, None, P, Q2, 1024, Q2, 256, None) == EINVAL
    for kw in (dict(q=None), dict(q=ODD), dict(qo=None), dict(qo=ODD), dict(k=None), dict(k=ODD), dict(ko=None), dict(ko=ODD), dict(cu=None), dict(cu=ODD), dict(pos=ODD),
               dict(f=None), dict(f=C.c_void_p(4100)), dict(qs=1016), dict(qs=1028), dict(qos=1016), dict(qos=1025), dict(ks=248), dict(kos=260), dict(qs=-1024),
               dict(q=Q2, qs=2048), dict(k=Q2, ks=512)):
        assert _rotary(_rs(), **kw) == EINVAL, kw
    assert _rotary(_rs(hkv=0)) == EINVAL                                            # keys without heads
    assert _rotary(_rs(n_tokens=0), q=None, k=None, cu=None, f=None, qo=None, ko=None) == OK


def _read(s, cu=P, n=P, t=P, kp=P, vp=P, ks=P, vs=P, k=Q2, kst=256, v=Q2, vst=256):
    return nsa.lib().nsa_sel_cache_read(C.byref(s), cu, n, t, kp, vp, ks, vs, k, kst, v, vst, None)


def test_read_refuses():
    base = dict(n_tokens=5, nseq=2, hq=8, hkv=2, dtype=1)
    for kw in (dict(n_tokens=-1), dict(nseq=-1), dict(nseq=0), dict(hkv=0), dict(hkv=3), dict(dtype=2), dict(n_pages=-1), dict(max_pages=-1)):
        assert _read(_shape(nsa, **{**base, **kw})) == EINVAL, kw
    for kw in (dict(d=64), dict(page=8), dict(page=48), dict(max_pages=2 ** 26), dict(n_tokens=2 ** 28)):
        assert _read(_shape(nsa, **{**base, **kw})) == UNSUPPORTED, kw
    s = _shape(nsa, **base)
    for kw in (dict(cu=None), dict(cu=ODD), dict(n=None), dict(n=ODD), dict(t=None), dict(t=ODD), dict(kp=None), dict(kp=ODD), dict(vp=None), dict(ks=None), dict(vs=ODD),
               dict(k=None), dict(k=ODD), dict(v=None), dict(v=ODD), dict(kst=248), dict(kst=260), dict(vst=0), dict(vst=-256)):
        assert _read(s, **kw) == EINVAL, kw
    assert _read(_shape(nsa, **{**base, "n_tokens": 0}), cu=None, n=None, t=None, kp=None, vp=None, k=None, v=None) == OK


def _chunk(s, q=P, cu=P, n=P, t=P, kp=P, vp=P, ks=P, vs=P, gate=None, acc=None, o=Q2, lse=P, ws=P, ws_bytes=1 << 40):
    return nsa.lib().nsa_sel_cache_attention_chunk(C.byref(s), q, cu, n, t, kp, vp, ks, vs, gate, acc, o, lse, ws, ws_bytes, None)


def _need(s):
    n = C.c_size_t(77)
    return nsa.lib().nsa_sel_cache_chunk_workspace_bytes(C.byref(s), C.byref(n)), n.value


def test_attention_of_pieces_refuses():
    base = dict(n_tokens=50, nseq=2, hq=8, hkv=2, dtype=1, topk=0)
    for kw in (dict(n_tokens=-1), dict(nseq=0), dict(hkv=3), dict(hq=18), dict(dtype=2), dict(window=-1), dict(topk=4)):
        s = _shape(nsa, **{**base, **kw})
        assert _chunk(s) == EINVAL and _need(s) == (EINVAL, 77), kw
    for kw in (dict(d=64), dict(page=8), dict(max_pages=2 ** 26), dict(topk=33)):
        s = _shape(nsa, **{**base, **kw})
        assert _chunk(s) == UNSUPPORTED and _need(s) == (UNSUPPORTED, 77), kw
    s = _shape(nsa, **base)
    rc, need = _need(s)
    assert rc == OK and need > 0
    for kw in (dict(q=None), dict(q=ODD), dict(cu=None), dict(cu=ODD), dict(n=None), dict(t=None), dict(kp=None), dict(vp=ODD), dict(ks=None), dict(vs=None), dict(o=None),
               dict(o=ODD), dict(o=P), dict(lse=None), dict(lse=ODD), dict(gate=ODD), dict(acc=P), dict(gate=P, acc=ODD), dict(ws=ODD)):
        assert _chunk(s, **kw) == EINVAL, kw
    assert _chunk(s, ws_bytes=need - 1) == WORKSPACE
    empty = _shape(nsa, **{**base, "n_tokens": 0})
    assert _need(empty) == (OK, 0)
    assert _chunk(empty, q=None, cu=None, n=None, t=None, kp=None, vp=None, o=None, lse=None, ws=None, ws_bytes=0) == OK


def test_workspace_of_the_largest_calls():
    """The launches do not grow with the call: the workspace is the same for every size."""
    sizes = {_need(_shape(nsa, topk=0, **kw)) for kw in (dict(n_tokens=1, nseq=1, hq=8, hkv=8), dict(n_tokens=(1 << 28) - 1, nseq=1, hq=8, hkv=1),
                                                        dict(n_tokens=1 << 24, nseq=1 << 24, hq=64, hkv=8), dict(n_tokens=(1 << 31) - 1, nseq=1 << 24, hq=1, hkv=1))}
    assert len(sizes) == 1 and sizes.pop()[0] == OK
    assert _need(_shape(nsa, n_tokens=1 << 28, nseq=1, hq=8, hkv=1, topk=0))[0] == UNSUPPORTED
    assert _need(_shape(nsa, n_tokens=1 << 25, nseq=(1 << 24) + 1, hq=1, hkv=1, topk=0))[0] == UNSUPPORTED


# ---- the Python calls ----------------------------------------------------------------------------------------------------------
def _cache(dtype=BF):
    return nsa.PagedCache(5, 2, page=64, dtype=dtype, device="cpu")


def _with(args, **kw):
    return {**args, **kw}


def test_python_read():
    cache = _cache()
    ok = dict(table=torch.zeros(3, 4, dtype=I32), kv_len=torch.ones(3, dtype=I32), cu=torch.zeros(4, dtype=I32), tokens=7)
    row = torch.zeros(7, 2, 128, dtype=BF)
    bad = [(_with(ok, table=ok["table"].long()), "table"), (_with(ok, table=ok["table"][:2]), "kv_len"), (_with(ok, kv_len=ok["kv_len"].float()), "kv_len"),
           (_with(ok, cu=ok["cu"][:3]), "cu_seqlens"), (_with(ok, tokens=None), "tokens"), (_with(ok, tokens=-1), "tokens"), (_with(ok, tokens=2 ** 40), "tokens"),
           (_with(ok, k_out=row[:6]), "tokens"), (_with(ok, tokens=None, k_out=row, v_out=row[:6].clone()), "v_out"), (_with(ok, k_out=row.float()), "k_out"),
           (_with(ok, k_out=torch.zeros(7, 2, 256, dtype=BF)[..., ::2]), "k_out"), (_with(ok, cu=None), "tokens"), (_with(ok, k_out=row.clone().requires_grad_()), "k_out requires")]
    for args, match in bad:
        with pytest.raises(nsa.NsaSelError, match=match):
            cache.read(**args)
    with pytest.raises(nsa.NsaSelError, match="device tensors"):                     # all that is wrong with the others
        cache.read(**ok)
    with pytest.raises(nsa.NsaSelError, match="device tensors"):
        cache.read(**_with(ok, tokens=None, k_out=row))


def test_python_attention_chunk():
    cache = _cache()
    q = torch.zeros(7, 8, 128, dtype=BF)
    ok = dict(q=q, table=torch.zeros(3, 4, dtype=I32), kv_len=torch.ones(3, dtype=I32), cu=torch.zeros(4, dtype=I32))
    gate = torch.zeros(7, 8)
    bad = [(_with(ok, q=q.float()), "q must be"), (_with(ok, q=q.transpose(0, 1).contiguous().transpose(0, 1)), "q must be contiguous"), (_with(ok, cu=None), "cu_seqlens"),
           (_with(ok, window=-1), "invalid"), (_with(ok, window=2 ** 31), "window"), (_with(ok, q=torch.zeros(7, 7, 128, dtype=BF)), "invalid"),
           (_with(ok, gate=gate[:6]), "gate"), (_with(ok, o_acc=q.clone()), "o_acc without gate"), (_with(ok, gate=gate, o_acc=q.float()), "o_acc"),
           (_with(ok, out=q[:6]), "out"), (_with(ok, lse=gate.double()), "lse"), (_with(ok, ws=torch.zeros(10, dtype=torch.uint8)), "ws holds"),
           (_with(ok, q=q.clone().requires_grad_()), "q requires grad"), (_with(ok, gate=gate.clone().requires_grad_()), "gate requires grad")]
    for args, match in bad:
        with pytest.raises(nsa.NsaSelError, match=match):
            cache.attention_chunk(**args)
    with pytest.raises(nsa.NsaSelError, match="device tensors"):
        cache.attention_chunk(**ok)
    assert cache.chunk_workspace_bytes(7, 8, 3, 4) > 0 and cache.chunk_workspace_bytes(0, 8, 3, 4) == 0
    for kw in (dict(tokens=2 ** 31), dict(window=2 ** 32), dict(max_pages=-2 ** 40)):
        with pytest.raises(nsa.NsaSelError, match="out of range"):
            cache.chunk_workspace_bytes(**_with(dict(tokens=7, hq=8, nseq=3, max_pages=4), **kw))


def test_python_rotary():
    q, k = torch.zeros(7, 8, 128, dtype=BF), torch.zeros(7, 2, 128, dtype=BF)
    f, _ = nsa.rotary_frequencies(64, device="cpu")
    ok = dict(q=q, k=k, inv_freq=f, cu=torch.zeros(4, dtype=I32))
    bad = [(_with(ok, q=None), "q must be"), (_with(ok, q=q.float()), "q must be"), (_with(ok, q=q[:6]), "k must have shape"), (_with(ok, k=k.half()), "k must be"),
           (_with(ok, q=torch.zeros(7, 8, 64, dtype=BF)), "q must have shape"), (_with(ok, q=q[:, :0]), "at least one head"), (_with(ok, inv_freq=f.float()), "inv_freq"),
           (_with(ok, inv_freq=f[:7]), "inv_freq"), (_with(ok, inv_freq=torch.zeros(72, dtype=torch.float64)), "inv_freq"), (_with(ok, cu=torch.zeros(4)), "cu_seqlens"),
           (_with(ok, cu=torch.zeros(1, dtype=I32)), "cu_seqlens"), (_with(ok, positions=torch.zeros(6, dtype=I32)), "positions"),
           (_with(ok, positions=torch.zeros(7, dtype=torch.int64)), "positions"), (_with(ok, factor=0.0), "factor"), (_with(ok, factor=float("nan")), "factor"),
           (_with(ok, q_out=q[:6]), "q_out"), (_with(ok, k=None, k_out=k), "k_out without k"), (_with(ok, q=torch.zeros(7, 8, 256, dtype=BF)[..., ::2]), "contiguous"),
           (_with(ok, q=torch.zeros(57, 128, dtype=BF).as_strided((7, 8, 128), (1, 128, 1))), "multiple of 8"),
           (_with(ok, q=torch.zeros(7 * 8 * 128 + 1, dtype=BF)[1:].view(7, 8, 128)), "aligned")]
    for args, match in bad:
        with pytest.raises(nsa.NsaSelError, match=match):
            nsa.rotary(**args)
    for args in (ok, _with(ok, k=None), _with(ok, cu=None), _with(ok, q=q.clone().requires_grad_())):
        with pytest.raises(nsa.NsaSelError, match="device tensors"):
            nsa.rotary(**args)
    with pytest.raises(nsa.NsaSelError, match="requires grad"):                       # a result that is given takes no gradient
        nsa.rotary(**_with(ok, q=q.clone().requires_grad_(), q_out=q.clone()))
    for grad in (q.clone().requires_grad_(), q):                                      # frequencies have no gradient
        with pytest.raises(nsa.NsaSelError, match="inv_freq requires grad"):
            nsa.rotary(**_with(ok, q=grad, inv_freq=f.clone().requires_grad_()))


def test_frequencies():
    f, a = nsa.rotary_frequencies(64, 10000.0, device="cpu")
    assert a == 1.0 and f.dtype == torch.float64 and torch.allclose(f, 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64), rtol=1e-15)
    assert torch.equal(nsa.rotary_frequencies(64, scaling="linear", stretch=4.0, device="cpu")[0], f / 4)
    g, _ = nsa.rotary_frequencies(64, scaling="base", stretch=4.0, device="cpu")
    assert g[0] == 1.0 and abs(float(g[-1] / f[-1]) - 0.25) < 1e-12 and bool((g.diff() < 0).all())
    h, a = nsa.rotary_frequencies(128, 500000.0, scaling="parts", stretch=8.0, trained=8192, device="cpu")
    whole, _ = nsa.rotary_frequencies(128, 500000.0, device="cpu")
    turns = 8192 * whole / (2 * torch.pi)
    assert torch.equal(h[turns >= 32], whole[turns >= 32]) and torch.allclose(h[turns <= 1], whole[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert bool((h[between] < whole[between]).all() and (h[between] > whole[between] / 8).all()) and abs(a - 1.2079441541679836) < 1e-15
    assert torch.equal(nsa.rotary_frequencies(64, scaling="parts", device="cpu")[0], f)
    for kw in (dict(rot=8), dict(rot=144), dict(rot=24), dict(base=1.0), dict(stretch=0.5), dict(fast=1.0), dict(trained=0), dict(scaling="other")):
        with pytest.raises(nsa.NsaSelError):
            nsa.rotary_frequencies(**kw, device="cpu")
