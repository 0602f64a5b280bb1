"""Batches over a paged cache for the tests: drawn on the host, uploaded, and compared with bounds that follow from the formats.

Bounds.  The kernels take bf16 products with fp32 sums, round each probability to bf16 (at most 2^-8 of it) and the result once more
(2^-8): |O - ref| <= 2^-8 sum(p |v|) + 2^-8 |ref|, and 2^-16 of the former for the fp32 sums and the base-2 exponentials, whose arguments
carry the error of a score.  A score of 128 products in fp32 is off by at most 128 * 2^-24 of the sum of its magnitudes S; LSE carries that, a
rounding of itself and the two functions: |LSE - ref| <= 2^-17 S + 2^-21 |ref| + 2^-20; a score's error also scales a probability: 2^-17 S more
of sum(p |v|)."""
import numpy as np
import torch

import workloads as wl

E4M3 = torch.float8_e4m3fn


def bf16(x):
    """float64 values that bf16 holds, from a normal draw."""
    return wl.bf16_bits_to_f64(wl.f32_to_bf16_bits(np.asarray(x, dtype=np.float32)))


def dev(x, dtype):
    if x is None:
        return None
    if dtype is E4M3:
        return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(E4M3).cuda()
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Batch:
    """Sequences of given lengths (new tokens included) over shuffled pages.  Everything that no sequence holds is NaN: pages that
    nobody has, slots behind a sequence's last token; table columns past a sequence's pages name no page or one that nobody has."""

    def __init__(self, seed, kv_len, new=None, *, hq=8, hkv=2, page=64, e4m3=False, pad=0, before=0, missing=(), spread=1.0):
        rng = self.rng = np.random.default_rng([20, seed])
        self.hq, self.hkv, self.page, self.e4m3 = hq, hkv, page, e4m3
        self.kv_len = np.array(kv_len, dtype=np.int32)
        n = len(kv_len)
        self.cu = None
        if new is not None:
            self.cu = (before + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
        self.T = n if new is None else int(self.cu[-1]) + pad
        need = [max(0, -(-int(L) // page)) for L in kv_len]
        self.n_pages = sum(need) + 3
        ids = rng.permutation(self.n_pages).astype(np.int32)
        width = max(need + [0]) + 2
        self.table = rng.choice(np.array([-1, self.n_pages, 2 ** 31 - 1, -2 ** 31, ids[-1]]), (n, width)).astype(np.int32)
        at = 0
        for s, c in enumerate(need):
            self.table[s, :c] = ids[at:at + c]
            at += c
        shape = (self.n_pages, hkv, page, 128)
        self.pages = [bf16(rng.standard_normal(shape) * spread) for _ in range(2)]
        self.scales = [None, None]
        if e4m3:
            self.pages = [np.where(np.abs(x) > 2 ** -9, x, 0.0) for x in self.pages]
            self.pages = [torch.from_numpy(np.clip(100 * x, -448, 448)).to(torch.float32).to(E4M3).to(torch.float64).numpy() for x in self.pages]
            self.scales = [2.0 ** rng.integers(-9, -4, shape[:2]).astype(np.float64) for _ in range(2)]
        self.live = np.zeros((self.n_pages, page), dtype=bool)
        for s in range(n):
            for u in range(max(0, int(kv_len[s]))):
                self.live[self.table[s, u // page], u % page] = True
        for x in self.pages:
            x[~self.live[:, None, :].repeat(hkv, 1)] = np.nan
        for s, c in missing:
            self.table[s, c] = -1
        self.q = bf16(rng.standard_normal((self.T, hq, 128)))
        self.k = bf16(rng.standard_normal((self.T, hkv, 128)))
        self.v = bf16(rng.standard_normal((self.T, hkv, 128)))

    def upload(self, nsa):
        t = E4M3 if self.e4m3 else torch.bfloat16
        f = torch.float32
        self.cache = nsa.PagedCache.from_tensors(*(dev(x, t) for x in self.pages), *(dev(x, f) for x in self.scales))
        self.dq, self.dk, self.dv = (dev(x, torch.bfloat16) for x in (self.q, self.k, self.v))
        self.dtable, self.dlen, self.dcu = (dev(x, torch.int32) for x in (self.table, self.kv_len, self.cu))
        return self.cache

    def draw_idx(self, topk, block):
        """Blocks by lot with repeats, padding, blocks of the future and beyond; some rows with nothing."""
        from oracle import paged_cache_oracle as pco
        idx = np.full((self.T, self.hkv, topk), -1, dtype=np.int32)
        for t, w in enumerate(pco.places(self.kv_len, self.cu, self.T)):
            cur = 0 if w is None else max(0, w[1] // block)
            idx[t] = self.rng.integers(-1, cur + 2, (self.hkv, topk))
            idx[t, :, 0] = cur
        idx[self.rng.random(idx.shape) < 0.03] = 2 ** 31 - 1
        if self.T > 2:
            idx[self.T // 2, 0] = -1
        return idx


def check_attention(o, lse, ref, gate=None, acc=None):
    """ref = the oracle's (O, LSE, A, S); rows of no sequence are not looked at."""
    O, LSE, A, S = ref
    o, lse = host(o), host(lse)
    on = ~np.isnan(LSE)
    assert np.array_equal(np.isneginf(lse[on]), np.isneginf(LSE[on]))
    fin = on & np.isfinite(LSE)
    err = np.abs(lse[fin] - LSE[fin])
    assert (err <= 2.0 ** -17 * S[fin] + 2.0 ** -21 * np.abs(LSE[fin]) + 2.0 ** -20).all(), err.max()
    own = (2.0 ** -8 + 2.0 ** -16 + 2.0 ** -17 * S[..., None]) * A
    if gate is not None:
        own, O = own * np.abs(gate)[..., None], gate[..., None] * O + (0.0 if acc is None else acc)
    err, allowed = np.abs(o - O), own + 2.0 ** -8 * (np.abs(O) + own)
    assert (err[on] <= allowed[on]).all(), float(np.nanmax(err[on] - allowed[on]))
