"""What a page loses when its scale grows: values of 2^-6 of the new scale and more are held exactly, smaller ones to half a step of the subnormal range."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grows", [1, 2, 5, 9])
def test_bounds_of_a_page_that_is_rounded_again(grows):
    """Every e4m3 value at scale 1, and then a token that makes the scale 2^grows."""
    every = torch.arange(256, dtype=torch.uint8).view(E4M3).to(torch.float64).numpy()
    every = np.where(np.isnan(every), 0.0, every)
    rows = every.reshape(2, 1, 128)                        # two tokens of a head; 448 is among them: scale 1
    cache = nsa.PagedCache(1, 1, page=16, dtype=E4M3)
    table, lens = dev([[0]], torch.int32), (lambda n: dev([n], torch.int32))
    x = dev(rows, torch.bfloat16)
    cache.append(x, x, table, lens(2), dev([0, 2], torch.int32))
    for pages, scale in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
        assert float(scale) == 1.0 and np.array_equal(host(pages[0, 0, :2]).reshape(2, 1, 128), rows)
    new = torch.full((1, 1, 128), 448.0 * 2.0 ** grows, dtype=torch.bfloat16, device="cuda")
    cache.append(new, new, table, lens(3))
    scale = 2.0 ** grows
    for pages, s in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
        assert float(s) == scale
        err = np.abs(host(pages[0, 0, :2]).reshape(2, 1, 128) * scale - rows)
        assert (err[np.abs(rows) >= 2.0 ** -6 * scale] == 0).all()
        assert err.max() <= 2.0 ** -10 * scale
        lossy = (np.abs(rows) < 2.0 ** -6 * scale) & (err > 0)
        assert lossy.any() and np.abs(rows)[lossy].max() > 2.0 ** -14 * scale
