"""The cache read back as rows, against the oracle's arrays: equal, since bf16 holds every stored value times its scale."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, Batch, dev, host
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


def _expected(b, x, scale):
    out = np.full((b.T, b.hkv, 128), np.nan)
    for t, w in enumerate(pco.places(b.kv_len, b.cu, b.T)):
        if w is None:
            continue
        at = pco.slot_of(b.table, b.n_pages, b.page, *w)
        out[t] = 0.0 if at is None else x[at[0], :, at[1]] * (1.0 if scale is None else scale[at[0], :, None])
    return out


def _check(b, k, v, untouched):
    for got, x, sc in zip((k, v), b.pages, b.scales):
        ref = _expected(b, x, sc)
        none = np.array([w is None for w in pco.places(b.kv_len, b.cu, b.T)], dtype=bool)
        assert np.array_equal(host(got)[~none], ref[~none], equal_nan=True)
        if untouched is not None:
            assert (host(got)[none] == untouched).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("hkv", [1, 2, 3, 8])
def test_rows(hkv, page, e4m3):
    """Whole sequences, their ends, none of one; tokens of no sequence; negative places and places without a page, which are zero."""
    b = Batch(81, [70, 33, 0, 300, 5, 1, 0], [70, 10, 0, 16, 9, 1, 2], hq=hkv, hkv=hkv, page=page, e4m3=e4m3, before=2, pad=4,
              missing=[(0, 0)] + ([(3, 18)] if page == 16 else []))
    cache = b.upload(nsa)
    fill = lambda: torch.full((b.T, hkv, 128), 5.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    k, v = fill(), fill()
    got = cache.read(b.dtable, b.dlen, b.dcu, k_out=k, v_out=v)
    assert got[0] is k and got[1] is v
    _check(b, k, v, 5.0)
    _check(b, *cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T), None)
    # into one tensor of both, whose tokens lie apart
    both = torch.full((b.T, 3 * hkv, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    cache.read(b.dtable, b.dlen, b.dcu, k_out=both[:, hkv:2 * hkv], v_out=both[:, 2 * hkv:])
    _check(b, both[:, hkv:2 * hkv], both[:, 2 * hkv:], 5.0)
    assert (both[:, :hkv] == 5).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_last_tokens_without_starts(e4m3):
    b = Batch(82, [70, 1, 0, 300], page=32, e4m3=e4m3)
    _check(b, *b.upload(nsa).read(b.dtable, b.dlen), None)


def test_every_value_of_8_bits_at_every_scale():
    """All 256 codes, NaN among them, times the largest and the smallest scale."""
    codes = torch.arange(256, dtype=torch.uint8).view(2, 1, 1, 128).expand(2, 1, 16, 128).contiguous()
    scale = torch.tensor([[2.0 ** -100], [2.0 ** 119]])
    cache = nsa.PagedCache.from_tensors(*(codes.cuda().view(E4M3) for _ in range(2)), *(scale.cuda() for _ in range(2)))
    table = torch.tensor([[0], [1], [1], [0]], dtype=torch.int32, device="cuda")
    k, v = cache.read(table, torch.full((4,), 3, dtype=torch.int32, device="cuda"))
    want = codes.view(E4M3).float() * scale.view(2, 1, 1, 1)
    want = want[[0, 1, 1, 0], :, 2].to(torch.bfloat16)
    for x in (k, v):
        assert torch.equal(x.cpu().nan_to_num(123.0), want.nan_to_num(123.0)) and torch.equal(x.cpu().isnan(), want.isnan())
        assert want.isnan().sum() == 4


def test_what_is_appended_is_read():
    rng = np.random.default_rng(83)
    lens = [40, 130, 7]
    cu = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), torch.int32)
    kv_len = dev(np.array(lens, dtype=np.int32), torch.int32)
    table = dev(rng.permutation(30).reshape(3, 10).astype(np.int32), torch.int32)
    k, v = (torch.randn(sum(lens), 2, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache = nsa.PagedCache(30, 2, page=16)
    f, _ = nsa.rotary_frequencies(64)
    _, turned = cache.append(k, v, table, kv_len, cu, inv_freq=f, rotated_k=True)
    got = cache.read(table, kv_len, cu, tokens=sum(lens))
    assert torch.equal(got[0], turned) and torch.equal(got[1], v)
    small = nsa.PagedCache(30, 2, page=16, dtype=E4M3)
    small.append(k, v, table, kv_len, cu)
    gk, gv = small.read(table, kv_len, cu, tokens=sum(lens))
    for x, y, sc in ((k, gk, small.k_scale), (v, gv, small.v_scale)):
        # half a step of the format: 2^-4 of the value, or of the smallest normal number of its page
        least = float(sc.max()) * 2.0 ** -6
        assert ((x.float() - y.float()).abs() <= 2.0 ** -4 * x.float().abs().clamp(min=least)).all()


def test_empty_reads():
    b = Batch(84, [50, 9], [10, 9], page=16)
    cache = b.upload(nsa)
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert cache.read(b.dtable, b.dlen, none, tokens=0)[0].shape == (0, 2, 128)
    k = torch.full((5, 2, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    cache.read(b.dtable, b.dlen, none, k_out=k)
    assert (k == 3).all()
    k, v = cache.read(b.dtable[:, :0].contiguous(), b.dlen, b.dcu, tokens=19)
    assert (k == 0).all() and (v == 0).all()
