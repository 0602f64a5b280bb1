"""Appending to pages in 8 bits where a workgroup takes several KV heads of a page, which share its angles: from 2 KV heads x pages that can be touched for each of 512
workgroups on (of 1024 in the form of 64 threads).  Batches of single tokens against the oracle, long prompts bit for bit against calls of fewer tokens, whose workgroups
take a head each."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, Batch, dev, host
from oracle import paged_cache_oracle as pco
from test_gpu_cache_append import _freq, _near, _run

pytestmark = pytest.mark.gpu


def _heads(units, hkv, threads):
    """KV heads of a workgroup, as the library's rule has them."""
    return min(max(units * hkv // (1024 if threads == 64 else 512), 1), hkv)


@pytest.mark.parametrize("n,hkv,page,heads", [(300, 8, 64, 2), (400, 8, 16, 3), (410, 5, 32, 2), (256, 8, 128, 2), (700, 3, 64, 2)])
def test_single_tokens_of_many_sequences(n, hkv, page, heads):
    """Pages that are empty, in part full and nearly full; some scales grow and some do not."""
    assert _heads(n, hkv, 64) == heads
    b = Batch(100 + n, [1 + (37 * i) % 90 for i in range(n)], hq=2 * hkv, hkv=hkv, page=page, e4m3=True)
    grow = np.exp2(np.arange(n) % 13 - 4.0)[:, None, None]
    b.k, b.v = b.k * grow, b.v * grow[::-1]
    _, old, new = _run(b, 128, False)
    held = [(b.table[s, L // page], L % page) for s, L in enumerate(b.kv_len - 1)]
    grew = [new[0][p] > old[0][p] for p, at in held if at > 0]
    assert 0.1 < np.mean(grew) < 0.9


@pytest.mark.parametrize("hkv,page", [(8, 64), (5, 32), (7, 256)])
def test_pages_of_several_tiles_in_place(hkv, page):
    """Single tokens in the mean, and sequences whose pages get more than the workgroup holds at once; the keys are their own results."""
    new = [200, 17, 70] + [1] * 300
    T, n = sum(new), len(new)
    assert _heads(T // page + 2 * n, hkv, 64) > 1
    b = Batch(120 + page, [230, 30, 70] + [1 + i % 60 for i in range(300)], new, hq=hkv, hkv=hkv, page=page, e4m3=True)
    pages, scales = [x.copy() for x in b.pages], [x.copy() for x in b.scales]
    f = _freq(128)
    turned = pco.append(b.k, b.v, b.table, b.kv_len, b.cu, pages, scales, page, f, False)
    cache = b.upload(nsa)
    cache.append(b.dk, b.dv, b.dtable, b.dlen, b.dcu, q=b.dq, inv_freq=dev(f, torch.float64), q_out=b.dq, k_out=b.dk)
    assert np.array_equal(host(cache.k_scale), scales[0]) and np.array_equal(host(cache.v_scale), scales[1])
    assert np.array_equal(host(cache.v_pages), pages[1], equal_nan=True)
    got, stored = host(b.dk), host(cache.k_pages)
    for t, (s, p) in enumerate(pco.places(b.kv_len, b.cu, T)):
        _near(got[t], turned[t], b.k[t], 2.0 ** -8)
        at = pco.slot_of(b.table, b.n_pages, page, s, p)
        unit = scales[0][at[0]][:, None]
        _near(stored[at[0], :, at[1]], turned[t] / unit, b.k[t] / unit, 2.0 ** -4, 2.0 ** -10)


@pytest.mark.parametrize("with_q", [False, True])
@pytest.mark.parametrize("lens,hkv,page,heads", [
    ([12000], 6, 64, 2),                                 # the query rows in the same launch
    ([20000, 37, 3000], 6, 64, 4),                       # in one of their own
    ([24000, 130], 11, 128, 4), ([9000, 15000, 1], 9, 16, 9),
    ([600] + [41] * 100, 8, 256, 3)])                    # few tokens a page in the mean, and pages of several tiles
def test_long_prompts_of_many_heads(lens, hkv, page, heads, with_q):
    rng = np.random.default_rng([121, page, hkv])
    T, n, hq = sum(lens), len(lens), hkv
    in_page = min(page, T // n)
    assert T >= 4096 and _heads(T // page + 2 * n, hkv, 512 if in_page > 64 else 256) == heads
    k, v = (torch.randn(T, hkv, 128, device="cuda").mul_(torch.rand(T, hkv, 1, device="cuda") * 8).bfloat16() for _ in range(2))
    q = torch.randn(T, hq, 128, device="cuda").bfloat16() if with_q else None
    per = [-(-L // page) for L in lens]
    ids = rng.permutation(sum(per))
    table = np.full((n, max(per)), -1)
    for s, c in enumerate(per):
        table[s, :c] = ids[sum(per[:s]):sum(per[:s + 1])]
    table = dev(table, torch.int32)
    f = dev(_freq(128, 500000.0), torch.float64)
    one, many = (nsa.PagedCache(sum(per), hkv, page=page, dtype=E4M3) for _ in range(2))
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    qo, ko = one.append(k, v, table, dev(lens, torch.int32), dev(cu, torch.int32), q=q, inv_freq=f, rotated_k=True)
    qs, ks = None if q is None else torch.full_like(qo, 7), torch.full_like(ko, 7)
    for s, L in enumerate(lens):
        for a in range(0, L, 1024):                        # whole pages a call
            c = min(1024, L - a)
            assert _heads(c // page + 2, hkv, 64 if min(page, c) <= 16 else 256) == 1
            rows = slice(int(cu[s]) + a, int(cu[s]) + a + c)
            many.append(k[rows], v[rows], table[s:s + 1], dev([a + c], torch.int32), dev([0, c], torch.int32), q=None if q is None else q[rows], inv_freq=f,
                        q_out=None if q is None else qs[rows], k_out=ks[rows])
    assert torch.equal(ko, ks) and (q is None or torch.equal(qo, qs))
    for x, y in ((one.k_pages, many.k_pages), (one.v_pages, many.v_pages), (one.k_scale, many.k_scale), (one.v_scale, many.v_scale)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
