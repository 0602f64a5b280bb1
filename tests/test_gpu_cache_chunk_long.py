"""Attention of pieces where a workgroup's part of a unit is longer than what it looks up of the page table at a time: 64 pieces, again from piece 61 of those on, and 64 in the pass that is
made again where values are not finite.  Against 64 bits on the device, with a bound on a row's norm that a wrong run of eight keys does not meet."""
import math

import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, dev

pytestmark = pytest.mark.gpu

# of csrc/cache_chunk.hip: what a unit costs beside its pieces, the least that a cut leaves, the most workgroups
UNIT_COST, LEAST_SPAN, WORKGROUPS = 6, 2, 256


def spans(pieces, heads):
    """Pieces of each workgroup's part of a unit, for units of these numbers of pieces, in order, of every KV head."""
    cost = [UNIT_COST + p for p in pieces] * heads
    share = -(-sum(cost) // WORKGROUPS)
    out, at = [], 0
    for c in cost:
        begin = 0
        for x in [*range((at // share + 1) * share - at, c, share), c]:
            end = c if x == c else 0 if x < UNIT_COST + LEAST_SPAN else c if x > c - LEAST_SPAN else x
            if end > begin:
                out.append(max(end - UNIT_COST, 0) - max(begin - UNIT_COST, 0))
                begin = end
        at += c
    return out


def row_norms(o, q, k, v, before, *, window=0, lse=None):
    """Of each row (n tokens of g heads behind `before` places; k, v [L, 128] in 64 bits): the norm of o's error, and that of what rounding makes of it.  A probability has 8 bits in its product: it
    is off by d_i of itself, so the row by sum d_i p_i v_i, whose square is, the d_i being independent, sum d_i^2 p_i^2 |v_i|^2 in the mean, with d^2 at most u^2 / 3 in the mean, u = 2^-8; the row
    itself is rounded to 8 bits once more.  (Sums, exponentials and scores in 32 bits add less than a hundredth of it.)  LSE, if it is given, is held to the bound of cache_util."""
    n, g = q.shape[:2]
    L = k.shape[0]
    scale = 1 / math.sqrt(128)
    rows = q.double().reshape(n * g, 128)
    at, place = torch.arange(L, device=q.device), before + torch.arange(n, device=q.device)
    on = at[None] <= place[:, None]
    if window:
        on &= at[None] > place[:, None] - window
    x = (torch.matmul(rows, k.T.contiguous()) * scale).view(n, g, L).masked_fill(~on[:, None], -math.inf)
    if lse is not None:
        ref = torch.logsumexp(x, -1)
        size = (torch.matmul(rows.abs(), k.abs().T.contiguous()) * scale).view(n, g, L).amax(-1)
        assert bool(((lse.double() - ref).abs() <= 2.0 ** -17 * size + 2.0 ** -21 * ref.abs() + 2.0 ** -20).all())
    p = torch.softmax(x, -1).view(n * g, L)
    want = torch.matmul(p, v).view(n, g, 128)
    rounding = 2.0 ** -8 / math.sqrt(3) * (torch.matmul(p.square(), v.square().sum(-1)).view(n, g) + want.square().sum(-1)).sqrt()
    return (o.double() - want).norm(dim=-1), rounding


class Shared:
    """Many sequences over pages that they share, each with its own pages for the new tokens; every table another order of them."""

    def __init__(self, seed, n, pieces_least, pieces_most, *, new=40, hkv=4, g=4, page=64, e4m3=False):
        rng = self.rng = np.random.default_rng([82, seed])
        self.n, self.hkv, self.g, self.page, self.new = n, hkv, g, page, new
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        full = rng.integers(pieces_least * 64 // page, pieces_most * 64 // page + 1, n)             # shared pages of a sequence
        pool, own = int(full.max()) + 40, (new + page - 1) // page + 1
        n_pages = pool + own * n
        order = rng.permutation(n_pages)
        self.table = np.full((n, int(full.max()) + own), -1, dtype=np.int32)
        for s in range(n):
            self.table[s, :full[s]] = order[rng.permutation(pool)[:full[s]]]
            self.table[s, full[s]:full[s] + own] = order[pool + own * s:pool + own * (s + 1)]
        self.kv_len = (full * page + rng.integers(new, new + page, n)).astype(np.int32)
        pages = [rand(n_pages, hkv, page, 128).to(torch.bfloat16) for _ in range(2)]
        scales = []
        if e4m3:
            pages = [(60 * x.float()).clamp(-448, 448).to(E4M3) for x in pages]
            scales = [2.0 ** torch.randint(-7, -4, (n_pages, hkv), generator=gen, device="cuda").float() for _ in range(2)]
        self.pages, self.scales = pages, scales
        self.q = rand(n * new, hkv * g, 128).to(torch.bfloat16)
        self.cu = np.arange(0, n * new + 1, new, dtype=np.int32)

    def run(self, **kw):
        cache = nsa.PagedCache.from_tensors(*self.pages, *self.scales)
        return cache.attention_chunk(self.q, dev(self.table, torch.int32), dev(self.kv_len, torch.int32), dev(self.cu, torch.int32), **kw)

    def rows(self, s, j):
        """K and V of sequence s, KV head j, in 64 bits."""
        u = torch.arange(int(self.kv_len[s]), device="cuda")
        page = torch.from_numpy(self.table[s]).cuda()[u // self.page].long()
        return [x[page, j, u % self.page].double() * (self.scales[i][page, j, None].double() if self.scales else 1.0) for i, x in enumerate(self.pages)]

    def spans(self, window=0):
        pieces = []
        for L in self.kv_len.tolist():
            first = max(L - self.new + 1 - window, 0) // 64 if window else 0
            pieces.append(-(-L // 64) - first)
        return spans(pieces, self.hkv)


def _check(b, o, lse, window=0, but=()):
    """Every row against 64 bits, those of a (sequence, KV head) among `but` left out.  A row's error is the sum of thousands of roundings, so its norm is near its mean, of which twice is allowed."""
    for s in range(b.n):
        tokens = slice(s * b.new, (s + 1) * b.new)
        for j in range(b.hkv):
            if (s, j) in but:
                continue
            heads = slice(j * b.g, (j + 1) * b.g)
            err, rounding = row_norms(o[tokens, heads], b.q[tokens, heads], *b.rows(s, j), int(b.kv_len[s]) - b.new, window=window, lse=lse[tokens, heads])
            assert bool((err <= 2 * rounding).all()), (s, j, float((err / rounding).max()))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 64])
def test_units_of_more_pieces_than_are_looked_up_at_once(page, e4m3):
    """Parts of more than 61 and of more than 122 pieces: pages are looked up twice and three times."""
    b = Shared(page + e4m3, 64, 100, 220, page=page, e4m3=e4m3)
    for window in (0, 64 * 150):
        of = b.spans(window)
        assert max(of) > 125 and sum(p > 122 for p in of) > 30 and sum(64 < p < 122 for p in of) > 10
        _check(b, *b.run(window=window), window=window)


@pytest.mark.parametrize("window", [0, 64 * 170])
@pytest.mark.parametrize("e4m3", [False, True])
def test_the_pass_that_is_made_again_looks_pages_up_too(e4m3, window):
    """A NaN in the key and the values of a later token: those that do not see it are as they are without it, over more than 64 pieces; and the other units are as they were."""
    b = Shared(7 + e4m3, 64, 180, 190, e4m3=e4m3)
    of = b.spans(window)
    assert sum(p > 64 for p in of) > 200 and sum(p > 128 for p in of) > 100
    bad, seen_by = {(s, s % b.hkv) for s in range(0, b.n, 3)}, 17                       # the last tokens, 17 of 40
    for s, j in bad:
        u = int(b.kv_len[s]) - seen_by
        for x in b.pages:
            bits = x.view(torch.uint8 if e4m3 else torch.int16)
            bits[int(b.table[s, u // b.page]), j, u % b.page, 7] = 0x7f if e4m3 else 0x7fc0
    o, lse = b.run(window=window)
    _check(b, o, lse, window, bad)
    for s, j in bad:
        L, heads = int(b.kv_len[s]), slice(j * b.g, (j + 1) * b.g)
        k, v = b.rows(s, j)
        assert bool(torch.isnan(k[L - seen_by]).any() and torch.isnan(v[L - seen_by]).any()) and int(torch.isnan(k).sum()) == 1
        before, after = slice(s * b.new, (s + 1) * b.new - seen_by), slice((s + 1) * b.new - seen_by, (s + 1) * b.new)
        n = b.new - seen_by
        err, rounding = row_norms(o[before, heads], b.q[before, heads], k[:L - seen_by], v[:L - seen_by], L - b.new, window=window, lse=lse[before, heads])
        assert err.shape[0] == n and bool((err <= 2 * rounding).all()), (s, j, float((err / rounding).max()))
        assert bool(torch.isnan(o[after, heads]).all()) and bool(torch.isnan(lse[after, heads]).all())
