"""Attention of pieces of prompts over a paged cache against 64 bits, element by element, with the bounds of cache_util (a probability rounded to bf16 is off by at most 2^-8 of
itself, which they count)."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch, bf16, check_attention, dev, host
from chunk_util import attend_chunks, check_chunks

pytestmark = pytest.mark.gpu


def _run(b, *, window=0, scale=0.0, gated=False, acc=True):
    cache = b.upload(nsa)
    out, lse = torch.full((b.T, b.hq, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((b.T, b.hq), 7.0, device="cuda")
    gate = b.rng.standard_normal((b.T, b.hq)).astype(np.float32) if gated else None
    o_acc = bf16(b.rng.standard_normal((b.T, b.hq, 128))) if gated and acc else None
    cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, window=window, scale=scale, gate=dev(gate, torch.float32), o_acc=dev(o_acc, torch.bfloat16), out=out, lse=lse)
    ref = attend_chunks(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, b.page, window=window, scale=scale)
    none = np.isnan(ref[1])
    if gated:
        gate = gate.astype(np.float64)
    check_chunks(out, lse, ref, gate, o_acc, keys=max(b.kv_len), most=np.nanmax(np.abs(b.pages[1])) * (1.0 if b.scales[1] is None else b.scales[1].max()))
    assert (host(lse)[none] == 7).all() and (host(out)[none] == 7).all()     # rows of no sequence are left as they were
    return out, lse


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (8, 8), (7, 1), (5, 1), (6, 2), (16, 2), (6, 3), (6, 1)])
def test_heads(hq, hkv, e4m3):
    """Every number of heads that share keys; a unit has 256 / g tokens, here more, fewer and exactly as many."""
    tok = 256 // (hq // hkv)
    _run(Batch(61, [tok + 40, 2 * tok + 3, 90], [tok, 2 * tok + 1, 33], hq=hq, hkv=hkv, page=32, e4m3=e4m3))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages_and_lengths(page, e4m3):
    """Lengths around pieces of 64 keys and pages, one token to many, sequences without new tokens, idle slots, tokens of no sequence before and behind."""
    _run(Batch(62, [1, 63, 64, 65, 0, 129, 300, 7, 256], [1, 63, 1, 2, 0, 100, 17, 0, 256], page=page, e4m3=e4m3, before=3, pad=5))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 100, 2 ** 31 - 1])
def test_windows(window, e4m3):
    _run(Batch(63, [400, 64, 130], [200, 64, 5], page=16, e4m3=e4m3), window=window)


@pytest.mark.parametrize("e4m3", [False, True])
def test_long_prefix(e4m3):
    """More than 64 pieces, whose pages are looked up in turns, and units that many workgroups share."""
    b = Batch(64, [9000, 4161, 70], [20, 70, 70], hq=4, hkv=1, page=64, e4m3=e4m3)
    _run(b)
    _run(b, window=4500)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("acc", [False, True])
def test_gated(acc, e4m3):
    _run(Batch(65, [500, 70], [90, 70], page=64, e4m3=e4m3, pad=1), gated=True, acc=acc, window=80)
    _run(Batch(65, [5000], [10], page=64, e4m3=e4m3), gated=True, acc=acc)     # joined from parts


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("e4m3", [False, True])
def test_missing_pages(window, e4m3):
    """Places without a page are invisible; rows that see nothing else are zero."""
    b = Batch(66, [200, 130, 40], [150, 64, 40], page=16, e4m3=e4m3, missing=[(0, 0), (0, 3), (0, 5), (0, 12), (1, 8), (2, 0), (2, 1), (2, 2)])
    out, lse = _run(b, window=window)
    assert np.isneginf(host(lse)[-40:]).all() and (host(out)[-40:] == 0).all()


def test_negative_places():
    """More new tokens than the length counts: those of negative place see nothing, whatever their query holds."""
    b = Batch(67, [30, 0, 100], [50, 3, 64], page=16)
    b.q[:5] = np.nan
    _run(b)
    _run(b, window=7)


def test_one_token_each_without_starts():
    _run(Batch(68, [1, 70, 0, 300, 4100], page=64))


@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_scores_near_and_far(spread):
    _run(Batch(69, [700, 90], [80, 90], page=64, spread=spread))
    _run(Batch(69, [700, 90], [80, 90], page=64, e4m3=True), scale=2.0)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("long", [False, True])
def test_what_a_token_does_not_see_does_not_matter(bad, long):
    """Infinities and NaN in the keys and values of a later token of the piece, before a window, and where a token sees them."""
    L, n = (6000, 90) if long else (150, 90)
    for window in (0, 40):
        b = Batch(70, [L, 64], [n, 64], hq=8, hkv=2, page=32)
        at = [L - n + 50, L - n + 51, L - n - 45 if not long else 5]
        for j, u in ((0, at[0]), (1, at[1]), (1, at[2]) if window else (1, at[1])):
            p = b.table[0, u // 32]
            b.pages[1][p, j, u % 32, 5] = bad
            b.pages[0][p, j, u % 32, 9] = bad if np.isnan(bad) else 0.0
        cache = b.upload(nsa)
        o, lse = (host(x) for x in cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, window=window))
        # the tokens that see none of it, against the same batch without it
        clean = [np.where(np.isfinite(x) | ~b.live[:, None, :, None], x, 0.0) for x in b.pages]
        ref = attend_chunks(b.q, b.table, b.kv_len, b.cu, clean, b.scales, 32, window=window)
        place = np.concatenate([np.arange(L - n, L), np.arange(64)])
        for j in range(2):
            mine = {u for k, u in ((0, at[0]), (1, at[1]), (1, at[2]) if window else (1, at[1])) if k == j}
            heads = slice(4 * j, 4 * j + 4)
            free = np.array([i >= n or not any(u <= p and (not window or u > p - window) for u in mine) for i, p in enumerate(place)])
            assert free.sum() >= 50 and (~free).sum() >= 10
            check_attention(torch.tensor(o[free][:, heads]), torch.tensor(lse[free][:, heads]), tuple(x[free][:, heads] for x in ref))
            assert not np.isfinite(o[~free][:, heads, 5]).any()
            if np.isnan(bad):
                assert np.isnan(lse[~free][:, heads]).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_many_units_of_many_sequences(e4m3):
    """More units than workgroups, of few pieces each; sequences without new tokens between."""
    rng = np.random.default_rng(5)
    new = [int(x) for x in rng.integers(0, 40, 150)]
    kv = [n + int(x) if n else int(x) for n, x in zip(new, rng.integers(0, 90, 150))]
    _run(Batch(71, kv, new, hq=8, hkv=4, page=16, e4m3=e4m3, pad=2))


def test_same_bits_again_and_in_parts_of_the_workspace():
    b = Batch(72, [3000, 500], [100, 300], page=64)
    cache = b.upload(nsa)
    need = cache.chunk_workspace_bytes(b.T, b.hq, 2, b.table.shape[1])
    got = []
    for fill in (0, 255):
        ws = torch.full((need + 100,), fill, dtype=torch.uint8, device="cuda")
        got.append(cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, ws=ws[:need]))
        assert (ws[need:] == fill).all()
    got.append(cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu))
    for o, l in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(l, got[0][1])
    # and as the attention of few tokens has it, up to both's roundings
    o, l = cache.attention(b.dq, b.dtable, b.dlen, b.dcu)
    ref = attend_chunks(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, b.page)
    check_attention(o, l, ref)


def test_empty_calls():
    b = Batch(73, [50, 9], [10, 9], page=16)
    cache = b.upload(nsa)
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    o, l = cache.attention_chunk(b.dq[:0], b.dtable, b.dlen, none)
    assert o.shape == (0, 8, 128) and l.shape == (0, 8)
    o, l = cache.attention_chunk(b.dq[:0], b.dtable[:0], b.dlen[:0])
    assert o.shape == (0, 8, 128)
    # tokens, but of no sequence
    out = torch.full((19, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    cache.attention_chunk(b.dq, b.dtable, b.dlen, none, out=out)
    assert (out == 3).all()
    # a table without columns: nothing is visible
    o, l = cache.attention_chunk(b.dq, b.dtable[:, :0].contiguous(), b.dlen, b.dcu)
    assert (o == 0).all() and torch.isneginf(l).all()
