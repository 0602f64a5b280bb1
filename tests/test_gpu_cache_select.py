"""Block selection for new tokens of cached sequences: bit for bit the oracle's."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
import workloads as wl
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu


def _scores(kind, T, hkv, stride, seed):
    rng = np.random.default_rng([21, seed])
    x = rng.standard_normal((T, hkv, stride)).astype(np.float32)
    if kind == "ties":
        x = np.round(x, 1)
    elif kind == "equal":
        x[:] = 0.25
    elif kind == "wild":
        x = np.exp(8 * x).astype(np.float32)
        x[rng.random(x.shape) < 0.1] = np.nan
        x[rng.random(x.shape) < 0.1] = -np.inf
        x[rng.random(x.shape) < 0.1] = np.inf
    return x


@pytest.mark.parametrize("kv,new,hkv,topk,block,n_sink,n_local,kind,stride", [
    ([1, 64, 65, 1000, 0], None, 2, 16, 64, 1, 2, "heavy", 16), ([2000] * 5, None, 3, 16, 64, 1, 2, "ties", 33),
    ([5000, 100], [3, 4], 1, 8, 128, 0, 1, "wild", 40), ([70000], None, 2, 16, 64, 1, 2, "heavy", 1096), ([131072, 66000, 40], [1, 2, 1], 2, 32, 64, 1, 2, "wild", 2048),
    ([300, 2], [2, 5], 2, 4, 64, 1, 1, "ties", 5), ([3000], None, 8, 12, 64, 0, 0, "equal", 47), ([640], None, 2, 8, 64, 1, 2, "heavy", 6),
    ([90000] * 3, None, 1, 31, 64, 2, 3, "equal", 1407), ([1000000], None, 2, 16, 64, 1, 2, "ties", 15628)])
def test_selection_bit_exact(kv, new, hkv, topk, block, n_sink, n_local, kind, stride):
    print("case", kv, new, hkv, topk, block, n_sink, n_local, kind, stride, flush=True)
    kv = np.array(kv, dtype=np.int32)
    cu = None if new is None else (1 + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
    T = len(kv) if new is None else int(cu[-1]) + 2
    x = _scores(kind, T, hkv, stride, stride)
    ref = pco.select(x, kv, cu, topk, block=block, n_sink=n_sink, n_local=n_local, untouched=-7)
    out = torch.full((T, hkv, topk), -7, dtype=torch.int32, device="cuda")
    got = nsa.select_blocks(torch.from_numpy(x).cuda(), None if cu is None else torch.from_numpy(cu).cuda(), topk, block=block, n_sink=n_sink,
                            n_local=n_local, kv_len=torch.from_numpy(kv).cuda(), out=out)
    assert got is out and np.array_equal(out.cpu().numpy(), ref)


def test_many_sequences():
    """More sequences than a wavefront has lanes, and than it has in two rounds; some without new tokens."""
    rng = np.random.default_rng(22)
    for n in (65, 5000):
        new = rng.integers(0, 3, n)
        kv = (new + rng.integers(0, 2000, n)).astype(np.int32)
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        x = _scores("ties", int(cu[-1]), 1, 32, n)
        got = nsa.select_blocks(torch.from_numpy(x).cuda(), torch.from_numpy(cu).cuda(), 6, kv_len=torch.from_numpy(kv).cuda())
        assert np.array_equal(got.cpu().numpy(), pco.select(x, kv, cu, 6))
