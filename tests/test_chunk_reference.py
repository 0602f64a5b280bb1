"""The reference of the chunk tests against the oracle of the cached calls, value by value; on the CPU."""
import numpy as np
import pytest

from cache_util import Batch
from chunk_util import attend_chunks
from oracle import paged_cache_oracle as pco


@pytest.mark.parametrize("kw", [dict(kv_len=[70, 5, 0, 33], new=[20, 5, 1, 0]), dict(kv_len=[40, 7], new=[40, 9], before=3, pad=2, e4m3=True),
                                dict(kv_len=[90, 3], new=[30, 2], missing=[(0, 1)], page=16), dict(kv_len=[9, 0, 50])])
@pytest.mark.parametrize("window,scale", [(0, 0.0), (17, 0.3)])
def test_against_the_oracle(kw, window, scale):
    b = Batch(7, **kw)
    got = attend_chunks(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, b.page, window=window, scale=scale)
    want = pco.attend(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, b.page, window=window, scale=scale)
    for x, y in zip(got, want):
        on = ~np.isnan(y)
        assert np.array_equal(on, ~np.isnan(x))
        assert np.array_equal(np.isneginf(x[on]), np.isneginf(y[on]))
        fin = on & np.isfinite(y)
        assert np.abs(x[fin] - y[fin]).max(initial=0.0) <= 1e-12 * max(1.0, np.abs(y[fin]).max(initial=0.0))
