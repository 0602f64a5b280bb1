"""Attention over a paged cache against the oracle in 64 bits, element by element, with bounds from the formats (cache_util)."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import Batch, check_attention, dev
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


def _run(b, idx=None, block=64, window=0, scale=0.0, gate=False, acc=False):
    print("case", b.kv_len[:9], None if b.cu is None else b.cu[:9], b.hq, b.hkv, "page", b.page, "e4m3", b.e4m3, "topk",
          None if idx is None else idx.shape[2], "block", block, "window", window, flush=True)
    cache = b.upload(nsa)
    ref = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, b.page, idx=idx, block=block, window=window, scale=scale)
    out = torch.full((b.T, b.hq, 128), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, b.hq), 55.0, device="cuda")
    gates = b.rng.random((b.T, b.hq)).astype(np.float32) if gate else None
    accs = b.q[::-1].copy() if acc else None
    o, l = cache.attention(b.dq, b.dtable, b.dlen, b.dcu, idx=dev(idx, torch.int32), block=block, window=window, scale=scale,
                           gate=dev(gates, torch.float32), o_acc=dev(accs, torch.bfloat16), out=out, lse=lse)
    torch.cuda.synchronize()
    assert o is out and l is lse
    check_attention(o, l, ref, None if gates is None else gates.astype(np.float64), accs)
    off = np.isnan(ref[1])
    assert (out.cpu()[torch.from_numpy(off)] == 77.0).all() and (lse.cpu()[torch.from_numpy(off)] == 55.0).all()
    return o, l


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,hq,hkv,page,topk,block", [
    ([1], 1, 1, 16, 1, 64), ([64], 8, 8, 64, 4, 64), ([65, 1, 300], 8, 2, 32, 5, 64), ([1000, 63, 128, 129], 28, 4, 64, 16, 64),
    ([777, 2000], 16, 2, 128, 32, 64), ([1500, 130, 0, 5], 10, 2, 256, 7, 128), ([700] * 9, 8, 1, 16, 8, 128), ([4000], 12, 4, 64, 16, 64)])
def test_selected_blocks_one_token_each(kv, hq, hkv, page, topk, block, e4m3):
    b = Batch(sum(kv) + topk, kv, hq=hq, hkv=hkv, page=page, e4m3=e4m3)
    _run(b, b.draw_idx(topk, block), block)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new,hq,hkv,page,window", [
    ([1], None, 4, 1, 64, 0), ([33, 64, 0, 1000], None, 8, 2, 16, 0), ([513, 100], None, 7, 1, 32, 100), ([2000], None, 8, 8, 256, 1),
    ([300, 20, 7], [5, 20, 0], 8, 2, 64, 0), ([300, 2, 700], [1, 4, 3], 16, 2, 32, 33), ([40, 90, 17, 130], [17, 1, 16, 31], 4, 4, 16, 20),
    ([5000], [7], 28, 4, 128, 0), ([260, 99], [40, 3], 3, 1, 64, 64)])
def test_every_key_and_windows(kv, new, hq, hkv, page, window, e4m3):
    b = Batch(sum(kv) + hq, kv, new, hq=hq, hkv=hkv, page=page, e4m3=e4m3, pad=0 if new is None else 3, before=0 if new is None else 2)
    _run(b, window=window)


@pytest.mark.parametrize("e4m3", [False, True])
def test_selected_blocks_of_several_tokens_with_gate_and_window(e4m3):
    b = Batch(5, [900, 70, 4, 333], [6, 9, 4, 0], hq=8, hkv=2, page=64, e4m3=e4m3, pad=2)
    idx = b.draw_idx(6, 64)
    _run(b, idx, gate=True)
    _run(b, idx, gate=True, acc=True)
    _run(b, idx, window=100, scale=0.25)


def test_many_rows_take_one_pass():
    """Enough rows that no row is split; the same tokens in a small batch are."""
    b = Batch(6, [500 + 7 * i for i in range(150)], hq=8, hkv=4, page=64)
    assert b.hkv * b.T > 512
    _run(b, b.draw_idx(4, 64))


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_do_not_exist(e4m3):
    """Columns of the table without a page, lengths beyond the table, more new tokens than the length says."""
    b = Batch(7, [400, 200, 90], [3, 2, 5], page=32, e4m3=e4m3, missing=((0, 0), (0, 5), (1, 6)))
    _run(b)
    _run(b, b.draw_idx(5, 64))
    b = Batch(8, [400, 200], page=16, e4m3=e4m3)
    b.table = b.table[:, :9].copy()
    _run(b)
    b = Batch(9, [100, 3], [2, 6], page=16, e4m3=e4m3)
    _run(b)
    b.kv_len[:] = [0, -5]
    _run(b)


def test_masked_values_of_any_kind_are_not_seen():
    """Keys and values of later tokens and before the window are NaN and infinite; tokens of a group see them differently."""
    b = Batch(10, [80, 50], [6, 4], hq=4, hkv=2, page=16)
    for s, n in ((0, 6), (1, 4)):
        u = int(b.kv_len[s]) - n // 2                 # the second half of the new tokens
        p, o = int(b.table[s, u // 16]), u % 16
        b.pages[0][p, :, o] = np.inf
        b.pages[1][p, :, o] = np.nan
        b.pages[1][p, :, o, ::2] = -np.inf
    ref = pco.attend(b.q, b.table, b.kv_len, b.cu, [np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0) for x in b.pages], b.scales, 16)
    cache = b.upload(nsa)
    o, l = cache.attention(b.dq, b.dtable, b.dlen, b.dcu)
    before = [0, 1, 2, 6, 7]
    check_attention(o[before], l[before], tuple(x[before] for x in ref))
    assert not torch.isfinite(o[[3, 4, 5, 8, 9]].float()).all(-1).any()
    # before the window
    b = Batch(11, [80], [6], hq=4, hkv=2, page=16)
    p, o = int(b.table[0, 50 // 16]), 50 % 16
    b.pages[0][p, :, o] = np.nan
    b.pages[1][p, :, o] = np.inf
    clean = [np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0) for x in b.pages]
    ref = pco.attend(b.q, b.table, b.kv_len, b.cu, clean, b.scales, 16, window=25)
    cache = b.upload(nsa)
    o, l = cache.attention(b.dq, b.dtable, b.dlen, b.dcu, window=25)
    rows = [1, 2, 3, 4, 5]                            # places 75 .. 79 see from 51 on, place 74 sees 50
    check_attention(o[rows], l[rows], tuple(x[rows] for x in ref))
    assert not torch.isfinite(o[0].float()).all(-1).any()


def test_scores_of_minus_infinity():
    """A row whose visible scores are all -inf is empty; single ones weigh nothing."""
    b = Batch(12, [70, 40], hq=2, hkv=1, page=16)
    b.q = np.abs(b.q) + 0.25
    b.q = np.asarray(b.q, dtype=np.float32).astype(np.float64)
    b.q = pco.to_bf16(b.q)
    b.pages[0][b.table[0, 2], :, 3:9, 0] = -np.inf
    for c in range(3):
        b.pages[0][b.table[1, c], :, :, 5] = np.where(np.isnan(b.pages[0][b.table[1, c], :, :, 5]), np.nan, -np.inf)
    with np.errstate(invalid="ignore"):
        O, LSE, A, S = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, 16)
        finite = pco.attend(b.q, b.table, b.kv_len, b.cu, [np.where(np.isinf(x), 0.0, x) for x in b.pages], b.scales, 16)
    cache = b.upload(nsa)
    o, l = cache.attention(b.dq, b.dtable, b.dlen)
    check_attention(o, l, (O, LSE, A, finite[3]))
    assert torch.isneginf(l[1]).all() and (o[1] == 0).all()


def test_a_large_cache_is_addressed_in_64_bits():
    """Pages past 4 GB and past 2^31 rows of a head: the same tokens at the far end and at the near end of a cache."""
    n_pages, hkv, page = 70000, 4, 64
    far = torch.empty(n_pages, hkv, page, 128, dtype=torch.bfloat16, device="cuda")
    far_v = torch.empty_like(far)
    b = Batch(13, [300, 100], hq=8, hkv=hkv, page=page)
    ref = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, page)
    b.upload(nsa)
    far[-b.n_pages:] = b.cache.k_pages
    far_v[-b.n_pages:] = b.cache.v_pages
    table = torch.where((b.dtable >= 0) & (b.dtable < b.n_pages), b.dtable + (n_pages - b.n_pages), b.dtable)
    o, l = nsa.PagedCache.from_tensors(far, far_v).attention(b.dq, table, b.dlen)
    check_attention(o, l, ref)


def test_results_do_not_depend_on_the_workspace_or_the_call():
    b = Batch(14, [3000, 100, 5], hq=8, hkv=2, e4m3=True)
    cache = b.upload(nsa)
    need = cache.workspace_bytes(3, 8, 3, b.table.shape[1])
    assert need > 0
    o, l = cache.attention(b.dq, b.dtable, b.dlen)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    o2, l2 = cache.attention(b.dq, b.dtable, b.dlen, ws=ws)
    assert torch.equal(o, o2) and torch.equal(l, l2)
    with pytest.raises(nsa.NsaSelError):
        cache.attention(b.dq, b.dtable, b.dlen, ws=ws[:need - 1])


def test_no_tokens():
    b = Batch(15, [30], hq=4, hkv=2)
    cache = b.upload(nsa)
    empty = torch.empty(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    o, l = cache.attention(empty, b.dtable[:0], b.dlen[:0])
    assert o.shape == (0, 4, 128) and l.shape == (0, 4)
    o, l = cache.attention(empty, b.dtable, b.dlen, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert o.shape == (0, 4, 128)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("kv,new,hq,hkv,page,window", [
    ([int(1.21 ** i) for i in range(1, 42)], None, 8, 4, 16, 0),                         # parts that end inside rows and span several
    ([2500, 3, 0, 1400, 77, 2000, 1, 1], [5, 3, 0, 2, 9, 1, 1, 0], 8, 2, 64, 0),         # the same with groups of tokens
    ([1 + 11 * (i % 7) for i in range(300)] + [1600], None, 4, 1, 32, 0),                # more sequences than threads
    ([3000, 1000, 1700], None, 4, 2, 16, 1500), ([2600, 90], [7, 30], 16, 2, 128, 1400), ([40000], None, 8, 1, 256, 0)])
def test_every_key_cut_evenly(kv, new, hq, hkv, page, window, e4m3):
    b = Batch(len(kv) + hq, kv, new, hq=hq, hkv=hkv, page=page, e4m3=e4m3, pad=0 if new is None else 2)
    assert b.table.shape[1] * page > 40 * 32 and (not window or window > 40 * 32)
    _run(b, window=window, gate=True)


@pytest.mark.parametrize("new", [None, [3, 9]])
def test_windows_longer_than_any_sequence(new):
    """They hide nothing, up to the longest that the argument holds; rows cut evenly, whole rows, selected blocks."""
    for kv in ([3000, 200], [300, 5]):  # of the latter's new tokens some have a negative place
        b = Batch(70 + kv[0], kv, new, hq=8, hkv=2, page=64)
        idx = b.draw_idx(4, 64)
        for window in (3001, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 16, 2 ** 31 - 1):
            _run(b, window=window)
            _run(b, idx, window=window)


def test_more_sequences_than_are_cut_evenly():
    """Every sequence is a workgroup's where a scan over the batch would cost more than it gives; a long table all the same."""
    b = Batch(41, [i % 50 for i in range(4100)] , hq=2, hkv=1, page=16)
    b.table = np.concatenate([b.table, np.full((4100, 100), -1, dtype=np.int32)], 1)
    _run(b)


def _shared(b, n, lens):
    """n sequences over the pages of the only one of `b`: prefixes of it."""
    rng = np.random.default_rng(42)
    b.table, b.kv_len = np.repeat(b.table, n, 0), np.array(lens, dtype=np.int32)
    b.T = n
    b.q = np.asarray(np.repeat(b.q, n, 0) * rng.choice([-1.0, -0.5, 0.5, 1.0], (n, b.hq, 128)))
    b.k, b.v = np.repeat(b.k, n, 0), np.repeat(b.v, n, 0)
    return b


@pytest.mark.parametrize("e4m3", [False, True])
def test_large_calls_over_shared_pages(e4m3):
    """Calls that read more than 96 MB, by which the reads are requested otherwise: selected blocks in parts, a window of many rows, every key."""
    rng = np.random.default_rng(43)
    b = _shared(Batch(44, [5000], hq=8, hkv=2, page=64, e4m3=e4m3), 60, [4100 + 15 * i for i in range(60)])
    idx = np.stack([np.stack([rng.permutation(32) for _ in range(2)]) for _ in range(60)]).astype(np.int32)
    _run(b, idx, block=128)
    b = _shared(Batch(45, [900], hq=8, hkv=4, page=32, e4m3=e4m3), 300, [1 + 3 * i for i in range(300)])
    assert 300 * 4 * 512 * 256 > 96 << 20
    _run(b, window=512)
    b = _shared(Batch(46, [3000], hq=8, hkv=4, page=64, e4m3=e4m3), 3, [3000, 64, 1234])
    b.table = np.concatenate([b.table, np.full((3, 1000), -1, dtype=np.int32)], 1)
    _run(b)


def test_random_calls():
    """Sizes, layouts, selections and windows by lot."""
    rng = np.random.default_rng(47)
    for i in range(40):
        hkv, g = int(rng.integers(1, 5)), int(rng.integers(1, 9))
        n = int(rng.integers(1, 9))
        kv = [int(rng.integers(0, 10 ** rng.integers(1, 4)) + 1) for _ in range(n)]
        new = [min(k, int(rng.integers(0, 12))) for k in kv] if rng.random() < 0.5 else None
        if new is not None and sum(new) == 0:
            new[0] = 1
        b = Batch(100 + i, kv, new, hq=hkv * g, hkv=hkv, page=int(rng.choice([16, 32, 64, 128, 256])), e4m3=bool(rng.random() < 0.5),
                  pad=0 if new is None else int(rng.integers(0, 3)), before=0 if new is None else int(rng.integers(0, 3)))
        block = int(rng.choice([64, 128]))
        _run(b, b.draw_idx(int(rng.integers(1, 33)), block) if rng.random() < 0.5 else None, block, window=int(rng.choice([0, 0, 1, 50, 700])),
             gate=bool(rng.random() < 0.3), acc=False, scale=float(rng.choice([0.0, 0.05])))
