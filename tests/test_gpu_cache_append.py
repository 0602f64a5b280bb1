"""Appending to a paged cache against the oracle in 64 bits.

Bounds: an angle is exact to 2^-24 turns of it and more, sine and cosine to 2^-23, the two products and their sum to 2^-23 of their
magnitudes: |y - ref| <= 2^-20 (|x_a| + |x_b|), then half a step of the format: 2^-8 |ref| in bf16; in e4m3, in units of the page's scale, 2^-4 |ref|
and at least 2^-10.  Values that are not rotated are stored exactly as the oracle stores them."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, Batch, bf16, dev, host
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


def _freq(rot, theta=10000.0):
    return None if rot == 0 else theta ** (-np.arange(0, rot, 2) / rot)


def _near(got, ref, x, half, least=0.0):
    """x: the values before the rotation, whose row's largest bounds |x_a| + |x_b|."""
    most = 2 * np.abs(x).max(-1, keepdims=True)
    err = np.abs(got - ref)
    allowed = 2.0 ** -20 * most + half * np.abs(ref) + least
    assert (err <= allowed * (1 + 2.0 ** -7)).all(), float((err - allowed).max())


def _run(b, rot, interleaved, slices=False):
    print("case", b.kv_len[:9], None if b.cu is None else b.cu[:9], b.hq, b.hkv, "page", b.page, "e4m3", b.e4m3, "rot", rot, interleaved, flush=True)
    f = _freq(rot)
    cache = b.upload(nsa)
    was = [x.view(torch.uint8).clone() for x in (cache.k_pages, cache.v_pages)]
    if slices:                                            # one projection's output, a token's heads side by side
        both = torch.full((b.T, b.hq + 2 * b.hkv + 1, 128), 9.0, dtype=torch.bfloat16, device="cuda")
        both[:, :b.hq], both[:, b.hq:b.hq + b.hkv], both[:, b.hq + b.hkv:-1] = b.dq, b.dk, b.dv
        b.dq, b.dk, b.dv = both[:, :b.hq], both[:, b.hq:b.hq + b.hkv], both[:, b.hq + b.hkv:-1]
    q_out = torch.full((b.T, b.hq, 128), 77.0, dtype=torch.bfloat16, device="cuda")
    k_out = torch.full((b.T, b.hkv, 128), 66.0, dtype=torch.bfloat16, device="cuda")
    got = cache.append(b.dk, b.dv, b.dtable, b.dlen, b.dcu, q=b.dq, inv_freq=dev(f, torch.float64), interleaved=interleaved, q_out=q_out,
                       k_out=k_out)
    torch.cuda.synchronize()
    assert got[0] is q_out and got[1] is k_out
    pages, scales = [x.copy() for x in b.pages], [None if x is None else x.copy() for x in b.scales]
    old_scales = [None if x is None else x.copy() for x in b.scales]
    turned = pco.append(b.k, b.v, b.table, b.kv_len, b.cu, pages, scales, b.page, f, interleaved)
    where = pco.places(b.kv_len, b.cu, b.T)
    # rows that leave
    for out, x, fill in ((q_out, b.q, 77.0), (k_out, b.k, 66.0)):
        out = host(out)
        for t, w in enumerate(where):
            if w is None or w[1] < 0:
                assert (out[t] == fill).all()
            elif f is None:
                assert np.array_equal(out[t], x[t], equal_nan=True)
            else:
                _near(out[t], pco.rotate(x[t], w[1], f, interleaved), x[t], 2.0 ** -8)
    # pages
    new = np.zeros((b.n_pages, b.page), dtype=bool)
    held = np.zeros((b.n_pages, b.page), dtype=bool)
    for t, w in enumerate(where):
        at = w and pco.slot_of(b.table, b.n_pages, b.page, *w)
        if at:
            new[at] = True
            rows = [(host(cache.k_pages[at[0], :, at[1]]), turned[t], pages[0], b.k[t], 0), (host(cache.v_pages[at[0], :, at[1]]), b.v[t], pages[1], b.v[t], 1)]
            for y, ref, stored, x, which in rows:
                if which == 1 or f is None:
                    assert np.array_equal(y, stored[at[0], :, at[1]], equal_nan=True)
                elif b.e4m3:
                    s = scales[0][at[0]][:, None]
                    _near(y, ref / s, x / s, 2.0 ** -4, 2.0 ** -10)
                else:
                    _near(y, ref, x, 2.0 ** -8)
    for p in range(b.n_pages):
        if new[p].any():
            held[p, :int(np.argmax(new[p]))] = True
    for i, x in enumerate((cache.k_pages, cache.v_pages)):
        now = x.view(torch.uint8)
        rest = torch.from_numpy(~(new | held))
        assert torch.equal(now.cpu().transpose(1, 2)[rest], was[i].cpu().transpose(1, 2)[rest])
        got_held, want_held = host(x).swapaxes(1, 2)[held], pages[i].swapaxes(1, 2)[held]
        assert np.array_equal(got_held, want_held, equal_nan=True)   # rounded again to a larger scale, or as they were
    if b.e4m3:
        assert np.array_equal(host(cache.k_scale), scales[0]) and np.array_equal(host(cache.v_scale), scales[1])
    return cache, old_scales, scales


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new,hq,hkv,page,rot,interleaved", [
    ([1], None, 1, 1, 16, 128, False), ([1000, 64, 65, 63, 1], None, 8, 2, 64, 128, False), ([300, 129, 128], None, 28, 4, 128, 64, True),
    ([50], [50], 8, 2, 16, 128, False), ([300, 70, 7, 64], [200, 70, 0, 1], 8, 2, 64, 128, True), ([700, 33], [651, 20], 4, 1, 256, 32, False),
    ([517, 40, 3], [300, 2, 3], 6, 3, 32, 96, False), ([100, 90], [30, 90], 8, 8, 64, 0, False), ([4100], [130], 2, 2, 128, 16, True)])
def test_append(kv, new, hq, hkv, page, rot, interleaved, e4m3):
    b = Batch(sum(kv) + rot, kv, new, hq=hq, hkv=hkv, page=page, e4m3=e4m3, pad=0 if new is None else 4, before=0 if new is None else 1)
    _run(b, rot, interleaved)


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_takes_slices_of_a_projection(e4m3):
    _run(Batch(31, [90, 20], [40, 20], hq=8, hkv=2, e4m3=e4m3), 128, False, slices=True)


def test_a_growing_scale_rounds_the_page_again():
    """Earlier tokens of a page are rounded to the larger scale, exactly as the oracle does; smaller new tokens leave it alone."""
    for factor in (2.0 ** 12, 2.0 ** 5, 2.0 ** -6):
        b = Batch(32, [40, 100, 61], hq=4, hkv=2, page=64, e4m3=True)
        b.k, b.v = b.k * factor, b.v * factor
        _, old, new = _run(b, 0, False)
        pages = [b.table[s, (n - 1) // 64] for s, n in enumerate((40, 100, 61))]
        grew = new[0][pages] > old[0][pages]
        assert grew.all() if factor > 1 else not grew.any()


def test_values_of_every_size():
    """Zeros, the least and the largest of bf16, infinities, NaN: scales stay normal, what is not finite is stored as NaN and does not count."""
    b = Batch(33, [5, 6, 7, 8, 9], hq=2, hkv=2, page=16, e4m3=True)
    b.kv_len[:] = 1
    b.k[0] = b.v[0] = 0.0
    b.k[1] = b.v[1] = 2.0 ** -133 * (np.arange(128) % 3)
    b.k[2] = b.v[2] = float(torch.finfo(torch.bfloat16).max) * np.where(np.arange(128) % 2, 1.0, -0.25)
    b.k[3, :, 7] = b.v[3, :, 9] = np.inf
    b.k[3, :, 8] = b.v[3, :, 1] = np.nan
    b.k[4] = b.v[4] = np.nan
    _run(b, 0, False)


def test_one_by_one_is_as_all_at_once():
    """A page filled token by token holds what one call writes, but for values that were rounded twice on the way into the subnormal range."""
    rng = np.random.default_rng(34)
    n, hkv = 64, 2
    k, v = (bf16(rng.standard_normal((n, hkv, 128)) * np.exp(rng.standard_normal((n, 1, 1)))) for _ in range(2))
    f = dev(_freq(128), torch.float64)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    one, all_ = (nsa.PagedCache(2, hkv, dtype=E4M3) for _ in range(2))
    dk, dv = dev(k, torch.bfloat16), dev(v, torch.bfloat16)
    for t in range(n):
        one.append(dk[t:t + 1], dv[t:t + 1], table, torch.tensor([t + 1], dtype=torch.int32, device="cuda"), inv_freq=f)
    all_.append(dk, dv, table, torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), inv_freq=f)
    for a, c, sa, sc in ((one.k_pages, all_.k_pages, one.k_scale, all_.k_scale), (one.v_pages, all_.v_pages, one.v_scale, all_.v_scale)):
        assert torch.equal(sa, sc)
        a, c = host(a[1]), host(c[1])
        assert np.array_equal(np.where(np.abs(c) >= 2.0 ** -6, a, 0), np.where(np.abs(c) >= 2.0 ** -6, c, 0))
        assert np.abs(a - c).max() <= 2.0 ** -9                # two half steps


def test_in_place_and_far_places():
    """q and k may be their own results; places around 2^20 lose nothing."""
    b = Batch(35, [2 ** 20 + 77], [3], hq=4, hkv=2, page=256)
    cache = b.upload(nsa)
    f = _freq(128, 500000.0)
    cache.append(b.dk, b.dv, b.dtable, b.dlen, b.dcu, q=b.dq, inv_freq=dev(f, torch.float64), q_out=b.dq, k_out=b.dk)
    for t in range(3):
        _near(host(b.dq[t]), pco.rotate(b.q[t], 2 ** 20 + 74 + t, f, False), b.q[t], 2.0 ** -8)
        _near(host(b.dk[t]), pco.rotate(b.k[t], 2 ** 20 + 74 + t, f, False), b.k[t], 2.0 ** -8)


@pytest.mark.parametrize("page", [64, 256])
def test_in_place_where_a_page_gets_more_than_the_mean(page):
    """Few new tokens in the mean and many in one sequence: its page is gone through twice, and the keys may be their own results."""
    new = [200] + [1] * 30
    b = Batch(39, [210] + [7] * 30, new, hq=4, hkv=2, page=page, e4m3=True)
    pages, scales = [x.copy() for x in b.pages], [x.copy() for x in b.scales]
    f = _freq(128)
    turned = pco.append(b.k, b.v, b.table, b.kv_len, b.cu, pages, scales, page, f, False)
    cache = b.upload(nsa)
    cache.append(b.dk, b.dv, b.dtable, b.dlen, b.dcu, q=b.dq, inv_freq=dev(f, torch.float64), q_out=b.dq, k_out=b.dk)
    for t, (s, p) in enumerate(pco.places(b.kv_len, b.cu, b.T)):
        _near(host(b.dk[t]), turned[t], b.k[t], 2.0 ** -8)
        _near(host(b.dq[t]), pco.rotate(b.q[t], p, f, False), b.q[t], 2.0 ** -8)
        at = pco.slot_of(b.table, b.n_pages, page, s, p)
        unit = scales[0][at[0]][:, None]
        _near(host(cache.k_pages[at[0], :, at[1]]), turned[t] / unit, b.k[t] / unit, 2.0 ** -4, 2.0 ** -10)
        assert np.array_equal(host(cache.v_pages[at[0], :, at[1]]), pages[1][at[0], :, at[1]])
    assert np.array_equal(host(cache.k_scale), scales[0]) and np.array_equal(host(cache.v_scale), scales[1])


def test_without_queries_and_without_tokens():
    b = Batch(36, [9, 30], hq=2, hkv=2, page=16)
    cache = b.upload(nsa)
    assert cache.append(b.dk, b.dv, b.dtable, b.dlen) == (None, None)
    assert np.array_equal(host(cache.k_pages)[b.table[1, 1], :, 13], b.k[1])
    cache.append(b.dk[:0], b.dv[:0], b.dtable[:0], b.dlen[:0])
    cache.append(b.dk[:0], b.dv[:0], b.dtable, b.dlen, torch.zeros(3, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_do_not_exist_are_not_written(e4m3):
    b = Batch(37, [100, 60], [50, 60], hq=2, hkv=2, page=16, e4m3=e4m3, missing=((0, 4), (1, 0), (1, 3)))
    _run(b, 64, False)
    b = Batch(38, [100, 5], [20, 9], hq=2, hkv=2, page=16, e4m3=e4m3)   # more new tokens than the length says
    _run(b, 64, False)
    b.table = b.table[:, :6].copy()                                       # a table that ends before the length
    _run(b, 64, False)


def test_random_appends():
    """Sizes, layouts, places and rotations by lot."""
    rng = np.random.default_rng(48)
    for i in range(30):
        hkv, g, n = int(rng.integers(1, 5)), int(rng.integers(1, 9)), int(rng.integers(1, 7))
        kv = [int(rng.integers(0, 10 ** rng.integers(1, 4)) + 1) for _ in range(n)]
        new = [min(k, int(rng.integers(0, 10 ** rng.integers(1, 3)))) for k in kv] if rng.random() < 0.6 else None
        if new is not None and sum(new) == 0:
            new[0] = 1
        b = Batch(200 + i, kv, new, hq=hkv * g, hkv=hkv, page=int(rng.choice([16, 32, 64, 128, 256])), e4m3=bool(rng.random() < 0.6),
                  pad=0 if new is None else int(rng.integers(0, 3)), before=0 if new is None else int(rng.integers(0, 3)))
        _run(b, 16 * int(rng.integers(0, 9)), bool(rng.random() < 0.4), slices=bool(rng.random() < 0.3))


@pytest.mark.parametrize("e4m3,page", [(False, 64), (True, 64), (True, 128), (True, 256)])
def test_long_prompts(e4m3, page):
    """From 4096 new tokens on rows and pages are gone through otherwise: heads share a page's angles, query rows are a launch of their own.  Against the
    same tokens in calls of whole pages and fewer tokens, which are held to the oracle: bit for bit."""
    rng = np.random.default_rng([49, page])
    lens = [6000, 37, 2500]
    hq, hkv, T = 12, 6, sum(lens)
    q, k, v = (torch.randn(T, h, 128, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    per = -(-max(lens) // page)
    table = dev(rng.permutation(3 * per).reshape(3, per), torch.int32)
    f = dev(_freq(128, 500000.0), torch.float64)
    one, many = (nsa.PagedCache(3 * per, hkv, page=page, dtype=E4M3 if e4m3 else torch.bfloat16) for _ in range(2))
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    qo, ko = one.append(k, v, table, dev(lens, torch.int32), dev(cu, torch.int32), q=q, inv_freq=f, rotated_k=True)
    qs, ks = torch.empty_like(qo), torch.empty_like(ko)
    for s, L in enumerate(lens):
        for a in range(0, L, 1024):                        # whole pages a call
            n = min(1024, L - a)
            rows = slice(int(cu[s]) + a, int(cu[s]) + a + n)
            many.append(k[rows], v[rows], table[s:s + 1], dev([a + n], torch.int32), dev([0, n], torch.int32), q=q[rows], inv_freq=f, q_out=qs[rows],
                        k_out=ks[rows])
    assert torch.equal(qo, qs) and torch.equal(ko, ks)
    assert torch.equal(one.k_pages.view(torch.uint8), many.k_pages.view(torch.uint8)) and torch.equal(one.v_pages.view(torch.uint8), many.v_pages.view(torch.uint8))
    if e4m3:
        assert torch.equal(one.k_scale, many.k_scale) and torch.equal(one.v_scale, many.v_scale)
