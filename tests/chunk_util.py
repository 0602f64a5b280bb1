"""Attention of pieces of prompts over a cache in 64 bits, a KV head of a sequence at a time (oracle/paged_cache_oracle.py goes token by token, which is too slow for long
ones); tests/test_chunk_reference.py pins it to that."""
import math

import numpy as np

from cache_util import host


def attend_chunks(q, table, kv_len, cu, pages, scales, page, *, window=0, scale=0.0):
    """(O, LSE, A, S) as paged_cache_oracle.attend without idx."""
    T, hq, d = q.shape
    n_pages, hkv = pages[0].shape[:2]
    g = hq // hkv
    scale = scale if scale > 0 else 1 / math.sqrt(d)
    O, LSE = np.full((T, hq, d), np.nan), np.full((T, hq), np.nan)
    A, S = np.zeros((T, hq, d)), np.zeros((T, hq))
    starts = range(len(kv_len) + 1) if cu is None else [int(x) for x in cu]
    for s in range(len(kv_len)):
        t0, n = starts[s], starts[s + 1] - starts[s]
        if n <= 0:
            continue
        places = int(kv_len[s]) - n + np.arange(n)
        L = max(0, min(int(kv_len[s]), table.shape[1] * page))
        u = np.arange(L)
        ids = table[s, u // page] if L else np.zeros(0, dtype=np.int64)
        there = (ids >= 0) & (ids < n_pages)
        ids = np.where(there, ids, 0)
        seen = there[None] & (u[None] <= places[:, None])
        if window:
            seen &= u[None] > places[:, None] - window
        for j in range(hkv):
            k, v = (x[ids, j, u % page] * (1.0 if sc is None else sc[ids, j, None]) for x, sc in zip(pages, scales))
            for i in range(n):
                at = np.flatnonzero(seen[i])
                rows = slice(j * g, (j + 1) * g)
                O[t0 + i, rows], LSE[t0 + i, rows] = 0.0, -np.inf
                if at.size == 0:
                    continue
                x = q[t0 + i, rows] @ k[at].T * scale
                S[t0 + i, rows] = (np.abs(q[t0 + i, rows]) @ np.abs(k[at]).T * scale).max(1)
                top = x.max(1, keepdims=True)
                if np.all(np.isneginf(top)):
                    continue
                with np.errstate(invalid="ignore"):
                    e = np.exp(x - top)
                    tot = e.sum(1, keepdims=True)
                    O[t0 + i, rows] = e @ v[at] / tot
                    A[t0 + i, rows] = e @ np.abs(v[at]) / tot
                LSE[t0 + i, rows] = (top + np.log(tot))[:, 0]
    return O, LSE, A, S


def check_chunks(o, lse, ref, gate=None, acc=None, keys=0, most=0.0):
    """cache_util.check_attention, whose bounds count relative errors only.  The largest probability of a row is 1, and one below 2^-126 is no normal number of 32 bits or bf16: the
    exponential and the matrix unit may take it as zero, which changes a result by at most 2^-126 |v|.  For `keys` keys with values up to `most` that is keys * 2^-126 * most."""
    O, LSE, A, S = ref
    o, lse = host(o), host(lse)
    on = ~np.isnan(LSE)
    assert np.array_equal(np.isneginf(lse[on]), np.isneginf(LSE[on]))
    fin = on & np.isfinite(LSE)
    err = np.abs(lse[fin] - LSE[fin])
    assert (err <= 2.0 ** -17 * S[fin] + 2.0 ** -21 * np.abs(LSE[fin]) + 2.0 ** -20).all(), err.max()
    own = (2.0 ** -8 + 2.0 ** -16 + 2.0 ** -17 * S[..., None]) * A + keys * 2.0 ** -126 * most
    if gate is not None:
        own, O = own * np.abs(gate)[..., None], gate[..., None] * O + (0.0 if acc is None else acc)
    err, allowed = np.abs(o - O), own + 2.0 ** -8 * (np.abs(O) + own)
    assert (err[on] <= allowed[on]).all(), float(np.nanmax(err[on] - allowed[on]))
