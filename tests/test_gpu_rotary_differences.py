"""The gradient of the rotation against differences, with a bound that a wrong gradient does not meet; and an input that wants none."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import bf16, dev, host
from test_gpu_rotary import _places, _turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [32, 128])
def test_gradient_against_differences(rot, interleaved):
    """<g, R(q + s) - R(q)> = <R^T g, s> for a linear R.  The step s lies along R^T g in 64 bits, 256 times as long, so that both sides are sums of squares and no sum of terms of any sign.  Every
    element of R(q + s), of R(q) and of the gradient is rounded once, at most 2^-8 of itself (and 2^-16 of the sizes in 32 bits): those, each times what it is multiplied by, bound the
    difference.  A gradient turned the wrong way, not turned, without the factor, or zero does not meet that bound."""
    rng = np.random.default_rng([94, rot])
    cu, T, factor = [0, 30, 31, 77], 80, 1.5
    q, g = (bf16(rng.standard_normal((T, 8, 128))) for _ in range(2))
    f = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    places = _places(cu, T)
    true = _turned(g, places, f, interleaved, factor, -1.0)[0]
    step = bf16(256 * true)
    args = dev(f, torch.float64), dev(np.array(cu, dtype=np.int32), torch.int32)
    far = bf16(q + step)
    step = far - q                                                                       # what the moved input is away by, exactly
    a = dev(q, torch.bfloat16).requires_grad_()
    y, _ = nsa.rotary(a, None, *args, interleaved=interleaved, factor=factor)
    y.backward(dev(g, torch.bfloat16))
    moved = host(nsa.rotary(dev(far, torch.bfloat16), None, *args, interleaved=interleaved, factor=factor)[0])
    by_difference = ((moved - host(y)) * g).sum()

    def allowed(grad):
        return (2.0 ** -8 + 2.0 ** -16) * ((np.abs(moved) * np.abs(g)).sum() + (np.abs(host(y)) * np.abs(g)).sum() + (np.abs(grad) * np.abs(step)).sum())

    grad = host(a.grad)
    assert abs(by_difference - (grad * step).sum()) <= allowed(grad)
    for wrong in (_turned(g, places, f, interleaved, factor, 1.0)[0], g * np.where(np.arange(128) < rot, factor, 1.0), _turned(g, places, f, interleaved, 1.0, -1.0)[0], 0 * g):
        assert abs(by_difference - (wrong * step).sum()) > allowed(wrong)


def test_an_input_without_a_gradient_takes_none():
    f, _ = nsa.rotary_frequencies(64)
    q, k = (torch.randn(40, h, 128, device="cuda").to(torch.bfloat16).requires_grad_() for h in (4, 2))
    a, b = nsa.rotary(q.detach(), k, f)
    assert b.requires_grad
    if a.requires_grad:                                                                   # of one node with b: nothing of it reaches k
        assert torch.autograd.grad(a.sum(), k, allow_unused=True)[0] is None
    leaf = q.detach()
    a, b = nsa.rotary(leaf, k, f)
    (a.float().sum() + b.float().sum()).backward()
    assert leaf.grad is None and torch.equal(k.grad, nsa.rotary(torch.ones_like(k), None, -f)[0].detach())
