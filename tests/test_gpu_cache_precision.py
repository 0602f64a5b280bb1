"""The attention's products of probabilities and values, where what a probability loses would show: long rows whose values cancel.

Bounds (with those of cache_util).  A probability goes into the product as the bf16 value below it and the rest, which is less than 2^-7 of it, as bf16: off by 2^-8
of the rest, 2^-15 of the probability.  2^-16 for the fp32 sums and the base-2 exponentials, 2^-17 S for a score's error: that much of
A = sum(p |v|).  The result is rounded once: |O - ref| <= own + 2^-8 (|O| + own), own = (2^-15 + 2^-16 + 2^-17 S) A.  Were a probability one bf16
value, it would be off by up to 2^-8 of itself, and a result near zero by much more than this."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch, check_attention, dev, host
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


def _check(b, idx=None, block=64, window=0, gate=False):
    print("case", b.kv_len[:9], None if b.cu is None else b.cu[:9], b.hq, b.hkv, "page", b.page, "e4m3", b.e4m3, "topk",
          None if idx is None else idx.shape[2], "block", block, "window", window, flush=True)
    b.q = b.q * 0.25                                      # scores below 2: no probability stands alone
    cache = b.upload(nsa)
    O, LSE, A, S = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, b.page, idx=idx, block=block, window=window)
    own = (2.0 ** -15 + 2.0 ** -16 + 2.0 ** -17 * S[..., None]) * A
    gates = accs = None
    if gate:
        gates, accs = b.rng.random((b.T, b.hq)).astype(np.float32), b.q[::-1].copy()
        own, O = own * gates[..., None].astype(np.float64), gates[..., None].astype(np.float64) * O + accs
    o, _ = cache.attention(b.dq, b.dtable, b.dlen, b.dcu, idx=dev(idx, torch.int32), block=block, window=window, gate=dev(gates, torch.float32),
                           o_acc=dev(accs, torch.bfloat16))
    on = ~np.isnan(LSE)
    err = np.abs(host(o) - O)[on]
    allowed = (own + 2.0 ** -8 * (np.abs(O) + own))[on]
    assert (err <= allowed).all(), (float((err / allowed).max()), float((err > allowed).mean()))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("kv,new,hq,hkv,topk,block,window", [
    ([1000, 700], None, 8, 1, 12, 64, 0), ([1900], None, 8, 2, 16, 64, 0), ([1500] * 4, None, 12, 4, 8, 128, 0),       # selected blocks
    ([900, 20], None, 7, 1, 0, 64, 300), ([3000, 50], None, 8, 2, 0, 64, 0), ([1100], None, 28, 4, 0, 64, 0),            # windows, every key, cut evenly
    ([900, 600], [7, 3], 8, 2, 0, 64, 0), ([1800, 90], [4, 9], 16, 2, 0, 64, 0), ([700], [5], 4, 4, 0, 64, 350)])         # tokens that share keys
def test_probabilities_keep_more_than_bf16_holds(kv, new, hq, hkv, topk, block, window, gate, e4m3):
    b = Batch(sum(kv) + hq + topk, kv, new, hq=hq, hkv=hkv, page=64, e4m3=e4m3)
    _check(b, b.draw_idx(topk, block) if topk else None, block, window, gate)


@pytest.mark.parametrize("kv,new", [([200], None), ([3000], None), ([200, 90], [3, 5])])
@pytest.mark.parametrize("selected", [False, True])
def test_infinite_values_that_are_seen(kv, new, selected):
    """A value of plus or minus infinity with a finite score makes its channel infinite, one of each NaN, as the sum over keys has it; the other channels
    are as they were.  A probability's parts may not make NaN of the former."""
    b = Batch(7 + sum(kv), kv, new, hq=8, hkv=2, page=64)
    for s in range(len(kv)):
        for u, c, x in ((3, 5, np.inf), (11, 70, -np.inf), (19, 9, np.inf), (40, 9, -np.inf)):
            b.pages[1][b.table[s, u // 64], :, u % 64, c] = x
    idx = b.draw_idx(3, 64) if selected else None
    if selected:
        idx[:, :, 1] = 0
    with np.errstate(invalid="ignore"):
        ref = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, 64, idx=idx)[0]
    cache = b.upload(nsa)
    o, _ = cache.attention(b.dq, b.dtable, b.dlen, b.dcu, idx=dev(idx, torch.int32))
    o = host(o)
    assert np.isposinf(ref[..., 5]).any() and np.isneginf(ref[..., 70]).any() and np.isnan(ref[..., 9]).any()
    for f in (np.isposinf, np.isneginf, np.isnan):
        assert np.array_equal(f(o), f(ref))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new", [([70], None), ([3000], None), ([70, 20], [3, 5])])
def test_an_empty_row_is_zero_whatever_its_values_are(kv, new, e4m3):
    """Every visible score is -inf: O = 0 (o_acc with a gate) and LSE = -inf, with values that are infinite or NaN too."""
    b = Batch(9 + sum(kv), kv, new, hq=4, hkv=1, page=64, e4m3=e4m3)
    b.q = pco.to_bf16(np.abs(b.q) + 0.25)
    if e4m3:                                              # no infinite key; a score of -inf comes from the query
        b.q[..., 5] = np.inf
        b.pages[0][..., 5] = np.where(np.isnan(b.pages[0][..., 5]), np.nan, -1.0)
    else:
        b.pages[0][..., 5] = np.where(np.isnan(b.pages[0][..., 5]), np.nan, -np.inf)
    b.pages[1][..., 9] = np.nan
    b.pages[1][..., 64] = np.nan if e4m3 else np.inf
    cache = b.upload(nsa)
    o, lse = cache.attention(b.dq, b.dtable, b.dlen, b.dcu)
    assert (o == 0).all() and torch.isneginf(lse).all()
    acc = torch.randn(b.T, 4, 128, device="cuda").bfloat16()
    o, lse = cache.attention(b.dq, b.dtable, b.dlen, b.dcu, gate=torch.rand(b.T, 4, device="cuda"), o_acc=acc)
    assert torch.equal(o, acc) and torch.isneginf(lse).all()


@pytest.mark.parametrize("kv,new", [([200], None), ([3000], None), ([200, 90], [3, 5])])
def test_large_values_without_weight(kv, new):
    """A key whose score is -inf, or far below the others, weighs nothing, with the largest finite value too."""
    b = Batch(11 + sum(kv), kv, new, hq=8, hkv=2, page=64)
    b.q = pco.to_bf16(np.abs(b.q) + 0.25)
    most = float(torch.finfo(torch.bfloat16).max)
    for s in range(len(kv)):
        for u, k, at in ((3, -np.inf, 5), (17, -np.inf, 5), (21, -1e20, 7), (40, -1e20, 64)):
            p = b.table[s, u // 64]
            b.pages[0][p, :, u % 64, at], b.pages[1][p, :, u % 64] = k, most * (-1) ** u
    for k in (3, 17, 21, 40):
        assert k < min(kv) - 8
    finite = [np.where(np.isinf(b.pages[0]), 0.0, b.pages[0]), b.pages[1]]
    with np.errstate(invalid="ignore"):
        O, LSE, A, S = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, 64)
    clean = [np.where(np.abs(x) > 1e19, 0.0, x) for x in finite]
    S = pco.attend(b.q, b.table, b.kv_len, b.cu, clean, b.scales, 64)[3]
    assert np.abs(O).max() < 100 and A.max() < 100        # those values are not in them
    o, lse = b.upload(nsa).attention(b.dq, b.dtable, b.dlen, b.dcu)
    check_attention(o, lse, (O, LSE, A, S))
