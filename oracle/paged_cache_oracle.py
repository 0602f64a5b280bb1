"""CPU oracle of the calls over a paged cache: append with rotation, attention, selection, in 64 bits.

TEST INFRASTRUCTURE ONLY: plain definitions, one token at a time, that share no code with the library.  tests/test_paged_cache_pins.py pins
them to the oracles of the training path, to closed forms and to torch's own 8-bit conversions.

A cache is a list of numpy arrays: pages [n_pages, hkv, page, d] of the values as stored (before a scale), scales [n_pages, hkv] or None.
New token i of n of sequence s has place kv_len[s] - n + i; cu None means one new token for each sequence.
"""
from __future__ import annotations

import math
from typing import Optional

import numpy as np

from oracle.topk_select_oracle import forced_blocks

E4M3_MAX = 448.0
SCALE_LEAST, SCALE_MOST = -100, 119


def places(kv_len, cu, T: int):
    """(sequence, place) of every token; None for tokens of no sequence."""
    if cu is None:
        return [(t, int(kv_len[t]) - 1) for t in range(T)]
    out = [None] * T
    for s in range(len(kv_len)):
        n = int(cu[s + 1]) - int(cu[s])
        for i in range(n):
            out[int(cu[s]) + i] = (s, int(kv_len[s]) - n + i)
    return out


def slot_of(table, n_pages: int, page: int, s: int, place: int):
    """(page id, slot) of a place, or None."""
    if place < 0 or place // page >= table.shape[1]:
        return None
    p = int(table[s, place // page])
    return (p, place % page) if 0 <= p < n_pages else None


def rotate(x: np.ndarray, place: int, inv_freq: Optional[np.ndarray], interleaved: bool) -> np.ndarray:
    """x [heads, d]."""
    y = np.array(x, dtype=np.float64)
    if inv_freq is None:
        return y
    n = len(inv_freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        c, s = math.cos(place * inv_freq[i]), math.sin(place * inv_freq[i])
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
    return y


def round_bits(x: np.ndarray, bits: int, least: float) -> np.ndarray:
    """Nearest value with `bits` significant bits, ties to even, steps of at least `least`."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.maximum(np.ldexp(1.0, e - bits), least)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(x), np.round(x / step) * step, x)


def to_bf16(x):
    return round_bits(x, 8, 0.0)


def to_e4m3(x):
    """Values already in a page's scale: saturated, rounded; infinities and NaN become NaN."""
    x = np.asarray(x, dtype=np.float64)
    y = round_bits(np.clip(np.where(np.isfinite(x), x, 0.0), -E4M3_MAX, E4M3_MAX), 4, 2.0 ** -9)
    return np.where(np.isfinite(x), y, np.nan)


def least_scale(x: np.ndarray) -> float:
    """Least power of two whose 448-fold holds all finite magnitudes."""
    a = np.abs(x[np.isfinite(x)])
    e = SCALE_LEAST
    while e < SCALE_MOST and a.size and a.max() > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(k, v, table, kv_len, cu, pages, scales, page: int, inv_freq=None, interleaved=False):
    """pages, scales: (K, V) each, updated in place.  Returns the rotated keys [T, hkv, d] in 64 bits (NaN where the token is not appended
    for having no sequence or a negative place)."""
    T, hkv, d = k.shape
    n_pages = pages[0].shape[0]
    where = places(kv_len, cu, T)
    turned = np.full(k.shape, np.nan)
    for t, w in enumerate(where):
        if w and w[1] >= 0:
            turned[t] = rotate(k[t], w[1], inv_freq, interleaved)
    per_page = {}
    for t, w in enumerate(where):
        at = w and slot_of(table, n_pages, page, *w)
        if at:
            per_page.setdefault(at[0], []).append((t, at[1]))
    for x, pg, sc in ((turned, pages[0], scales[0]), (v, pages[1], scales[1])):
        for p, rows in per_page.items():
            for j in range(hkv):
                if sc is None:
                    for t, slot in rows:
                        pg[p, j, slot] = to_bf16(x[t, j])
                    continue
                new = least_scale(np.stack([x[t, j] for t, _ in rows]))
                held = min(slot for _, slot in rows)
                if held > 0:
                    old = float(sc[p, j])
                    new = max(new, old)
                    pg[p, j, :held] = to_e4m3(pg[p, j, :held] * (old / new))
                for t, slot in rows:
                    pg[p, j, slot] = to_e4m3(x[t, j] / new)
                sc[p, j] = new
    return turned


def attend(q, table, kv_len, cu, pages, scales, page: int, *, idx=None, block=64, window=0, scale=0.0):
    """(O, LSE, A, S) with A = sum of p |v| and S = the largest sum of |q_i k_i| * scale over a row's visible keys: what errors are measured against.  NaN
    rows: tokens of no sequence."""
    T, hq, d = q.shape
    n_pages, hkv = pages[0].shape[:2]
    g = hq // hkv
    scale = scale if scale > 0 else 1 / math.sqrt(d)
    O, LSE = np.full((T, hq, d), np.nan), np.full((T, hq), np.nan)
    A, S = np.zeros((T, hq, d)), np.zeros((T, hq))
    for t, w in enumerate(places(kv_len, cu, T)):
        if w is None:
            continue
        s, p = w
        for j in range(hkv):
            if idx is None:
                keys = range(0, p + 1)
            else:
                kept = sorted({int(b) for b in idx[t, j] if 0 <= int(b) * block <= p})
                keys = [u for b in kept for u in range(b * block, min((b + 1) * block, p + 1))]
            at = [slot_of(table, n_pages, page, s, u) for u in keys if not window or u > p - window]
            at = [a for a in at if a]
            rows = slice(j * g, (j + 1) * g)
            if not at:
                O[t, rows], LSE[t, rows] = 0.0, -np.inf
                continue
            ids, slots = np.array([a[0] for a in at]), np.array([a[1] for a in at])
            k, v = pages[0][ids, j, slots].astype(np.float64), pages[1][ids, j, slots].astype(np.float64)
            if scales[0] is not None:
                k, v = k * scales[0][ids, j, None], v * scales[1][ids, j, None]
            x = q[t, rows] @ k.T * scale
            S[t, rows] = (np.abs(q[t, rows]) @ np.abs(k).T * scale).max(1)
            top = x.max(1, keepdims=True)
            if np.all(np.isneginf(top)):
                O[t, rows], LSE[t, rows] = 0.0, -np.inf
                continue
            e = np.exp(x - top)
            tot = e.sum(1, keepdims=True)
            O[t, rows] = e @ v / tot
            A[t, rows] = e @ np.abs(v) / tot
            LSE[t, rows] = (top + np.log(tot))[:, 0]
    return O, LSE, A, S


def select(scores, kv_len, cu, topk: int, *, block=64, n_sink=1, n_local=2, untouched=-1):
    T, hkv, stride = scores.shape
    out = np.full((T, hkv, topk), untouched, dtype=np.int32)
    for t, w in enumerate(places(kv_len, cu, T)):
        if w is None:
            continue
        cur = w[1] // block if w[1] >= 0 else -1
        b_vis = min(cur + 1, stride)
        for j in range(hkv):
            forced = forced_blocks(cur, b_vis, n_sink, n_local)[:topk]
            free = [b for b in range(b_vis) if b not in forced]
            free.sort(key=lambda b: (math.inf if math.isnan(scores[t, j, b]) else -float(scores[t, j, b]), b))
            sel = forced + free[:topk - len(forced)]
            out[t, j] = sel + [-1] * (topk - len(sel))
    return out
