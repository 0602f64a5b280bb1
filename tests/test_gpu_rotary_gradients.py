"""Gradients of the rotation that come out of a flat buffer."""
import pytest
import torch

import paper_2508_18224_amd as nsa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("ahead", [1, 4, 7, 8, 12])
def test_gradients_that_lie_anywhere_in_a_buffer(ahead, tokens):
    """What torch.cat hands back is a slice of its own gradient: contiguous, `ahead` values behind an aligned address.  For q, for k, and for both."""
    f, factor = nsa.rotary_frequencies(64, scaling="parts", stretch=4.0)
    q, k = (torch.randn(tokens, h, 128, device="cuda").to(torch.bfloat16).requires_grad_() for h in (4, 2))
    g = torch.randn(ahead + tokens * 6 * 128, device="cuda").to(torch.bfloat16)
    first = torch.zeros(ahead, dtype=torch.bfloat16, device="cuda")
    gq, gk = g[ahead:ahead + tokens * 512].clone().view(tokens, 4, 128), g[ahead + tokens * 512:].clone().view(tokens, 2, 128)
    want = nsa.rotary(gq, gk, -f, factor=factor)
    for of in ("q", "k", "both"):
        a, b = nsa.rotary(q, k, f, factor=factor)
        parts = [first] + ([a.flatten()] if of != "k" else []) + ([b.flatten()] if of != "q" else [])
        seed = g if of == "both" else torch.cat([first, (gq if of == "q" else gk).flatten()])
        got = torch.autograd.grad(torch.cat(parts), (q, k), seed, allow_unused=True)
        for x, w, there in zip(got, want, (of != "k", of != "q")):
            assert torch.equal(x, w) if there else x is None
