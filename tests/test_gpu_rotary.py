"""Rotary positions of the training path: against 64 bits, against the append to a cache (same bits), gradients against the transpose and against differences.

Bound.  A result is the sum of two products in 32 bits of bf16 values and a cosine or sine that is rounded once: 2^-24 of each product for that, 2^-24 for the product and
2^-24 of the sum, so at most 4 * 2^-24 (|x_a| + |x_b|) factor, and half a step of bf16, 2^-8 of the result.  The angle in 64 bits is off by 2^-50 of itself at most, below
2^-24 where places are below 2^20."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import bf16, dev, host

pytestmark = pytest.mark.gpu


def _turned(x, place, f, interleaved, factor=1.0, sign=1.0):
    """x [T, heads, 128], place [T] (None: copied) in 64 bits, and the bound's |x_a| + |x_b|."""
    y, size = x.copy(), np.abs(x)
    n = len(f)
    for t, p in enumerate(place):
        if p is None:
            continue
        a, b = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
        c, s = np.cos(p * f), sign * np.sin(p * f)
        u, v = x[t][:, a], x[t][:, b]
        y[t][:, a], y[t][:, b] = factor * (u * c - v * s), factor * (v * c + u * s)
        size[t][:, a] = size[t][:, b] = factor * (np.abs(u) + np.abs(v))
    return y, size


def _close(got, ref):
    y, size = ref
    err = np.abs(host(got) - y)
    assert (err <= 2.0 ** -8 * np.abs(y) + 4 * 2.0 ** -24 * size).all(), err.max()


def _places(cu, T):
    out = [None] * T
    for s in range(len(cu) - 1):
        for i in range(cu[s + 1] - cu[s]):
            out[cu[s] + i] = i
    return out


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 64, 96, 128])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (1, 0), (5, 1), (28, 4), (64, 8), (3, 3)])
def test_forward(hq, hkv, rot, interleaved):
    """Packed sequences, empty ones among them, tokens of no sequence at both ends; every number of rows to a workgroup; factor."""
    rng = np.random.default_rng([91, hq, rot])
    cu = [2, 2, 40, 41, 41, 130]
    T = 133
    q, k = bf16(rng.standard_normal((T, hq, 128))), bf16(rng.standard_normal((T, max(hkv, 1), 128)))
    f = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    for factor in (1.0, 1.25):
        a, b = nsa.rotary(dev(q, torch.bfloat16), dev(k, torch.bfloat16) if hkv else None, dev(f, torch.float64), dev(np.array(cu, dtype=np.int32), torch.int32),
                          interleaved=interleaved, factor=factor)
        _close(a, _turned(q, _places(cu, T), f, interleaved, factor))
        if hkv:
            _close(b, _turned(k, _places(cu, T), f, interleaved, factor))
        else:
            assert b is None
        for t in (0, 1, 130, 132):
            assert np.array_equal(host(a)[t], q[t])                      # of no sequence: copied


@pytest.mark.parametrize("interleaved", [False, True])
def test_places_that_are_given(interleaved):
    """Far ones, negative ones, in any order; starts beside them are not looked at."""
    rng = np.random.default_rng(92)
    place = rng.integers(-2 ** 20, 2 ** 20, 77).astype(np.int32)
    q, k = bf16(rng.standard_normal((77, 4, 128))), bf16(rng.standard_normal((77, 2, 128)))
    f = 500000.0 ** (-np.arange(0, 128, 2) / 128)
    for cu in (None, torch.zeros(3, dtype=torch.int32, device="cuda")):
        a, b = nsa.rotary(dev(q, torch.bfloat16), dev(k, torch.bfloat16), dev(f, torch.float64), cu, positions=dev(place, torch.int32), interleaved=interleaved)
        _close(a, _turned(q, place.tolist(), f, interleaved))
        _close(b, _turned(k, place.tolist(), f, interleaved))


@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True), (32, False)])
def test_same_bits_as_the_append(rot, interleaved):
    lens = [70, 1, 33]
    T = sum(lens)
    cu = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), torch.int32)
    q, k = (torch.randn(T, h, 128, device="cuda").to(torch.bfloat16) for h in (8, 2))
    f, _ = nsa.rotary_frequencies(rot)
    cache = nsa.PagedCache(24, 2, page=16)
    table = torch.arange(24, dtype=torch.int32, device="cuda").view(3, 8)
    a, b = cache.append(k, k, table, cu.diff(), cu, q=q, inv_freq=f, interleaved=interleaved, rotated_k=True)
    x, y = nsa.rotary(q, k, f, cu, interleaved=interleaved)
    assert torch.equal(a, x) and torch.equal(b, y)


def test_slices_and_results_in_place():
    T = 50
    f, _ = nsa.rotary_frequencies(128)
    x = torch.randn(T, 12, 128, device="cuda").to(torch.bfloat16)
    want = nsa.rotary(x[:, :8].contiguous(), x[:, 8:10].contiguous(), f)
    got = nsa.rotary(x[:, :8], x[:, 8:10], f)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q, k, rest = x[:, :8], x[:, 8:10], x[:, 10:].clone()
    out = nsa.rotary(q, k, f, q_out=q, k_out=k)                              # in the projection itself
    assert out[0] is q and torch.equal(x[:, :8], want[0]) and torch.equal(x[:, 8:10], want[1]) and torch.equal(x[:, 10:], rest)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [32, 128])
def test_gradients(rot, interleaved):
    """The gradient is the transpose: against 64 bits, and <g, R e> for a step e against <R^T g, e> and the difference of two forward passes."""
    rng = np.random.default_rng([93, rot])
    cu, T = [0, 30, 31, 77], 80
    q, k, gq, gk, e = (bf16(rng.standard_normal((T, h, 128))) for h in (8, 2, 8, 2, 8))
    f = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    dq, dk = dev(q, torch.bfloat16).requires_grad_(), dev(k, torch.bfloat16).requires_grad_()
    args = dev(f, torch.float64), dev(np.array(cu, dtype=np.int32), torch.int32)
    a, b = nsa.rotary(dq, dk, *args, interleaved=interleaved, factor=1.5)
    torch.autograd.backward((a, b), (dev(gq, torch.bfloat16), dev(gk, torch.bfloat16)))
    for got, g in ((dq.grad, gq), (dk.grad, gk)):
        _close(got, _turned(g, _places(cu, T), f, interleaved, 1.5, -1.0))
    # the forward pass is linear: a large step takes the roundings out of the difference
    moved, _ = nsa.rotary(dev(q + 256 * e, torch.bfloat16).detach(), None, *args, interleaved=interleaved, factor=1.5)
    step = host(dev(q + 256 * e, torch.bfloat16)) - q
    by_difference = ((host(moved) - host(a)) * gq).sum()
    by_gradient = (host(dq.grad) * step).sum()
    size = (np.abs(host(moved)) * np.abs(gq)).sum() + (np.abs(host(a)) * np.abs(gq)).sum() + (np.abs(host(dq.grad)) * np.abs(step)).sum()
    assert abs(by_difference - by_gradient) <= 2.0 ** -7 * size


def test_gradients_that_come_as_autograd_made_them():
    """Expanded, transposed, missing; one input alone; of slices of one projection; twice."""
    f, _ = nsa.rotary_frequencies(64)
    x = torch.randn(40, 6, 128, device="cuda").to(torch.bfloat16)
    q, k = x[:, :4].detach().requires_grad_(), x[:, 4:].detach().requires_grad_()
    ones = torch.ones(40, 4, 128, dtype=torch.bfloat16, device="cuda")
    back = lambda g: nsa.rotary(g, None, -f)[0]  # noqa: E731
    a, b = nsa.rotary(q, k, f)
    assert torch.equal(torch.autograd.grad(a.sum(), q)[0], back(ones))                # expanded, and nothing for k
    a, b = nsa.rotary(q, k, f)
    g = torch.randn(2, 40, 128, device="cuda").to(torch.bfloat16)
    assert torch.equal(torch.autograd.grad(b.transpose(0, 1), k, g)[0], back(g.transpose(0, 1).contiguous()))
    a, b = nsa.rotary(q.detach(), k, f)
    assert not a.requires_grad or a.grad_fn is not None
    assert torch.autograd.grad(b.sum(), k)[0].shape == k.shape
    w = x.clone().requires_grad_()
    a, b = nsa.rotary(w[:, :4], w[:, 4:], f)
    (a.float().sum() + 2 * b.float().sum()).backward()
    assert torch.equal(w.grad[:, :4], back(ones)) and torch.equal(w.grad[:, 4:], back(2 * ones[:, :2]))
    q2 = q.detach().requires_grad_()
    a, _ = nsa.rotary(q2, None, f)
    (d,) = torch.autograd.grad(a, q2, ones.requires_grad_(), create_graph=True)
    (dd,) = torch.autograd.grad(d, ones, q2.detach())
    assert torch.equal(dd, nsa.rotary(q2.detach(), None, f)[0])                        # the transpose of the transpose


def test_a_training_step_with_selected_attention():
    """Rotation, selected attention and its backward: as with the rotation taken apart."""
    T, HQ, HKV = 300, 8, 2
    q, k, v = (torch.randn(T, h, 128, device="cuda").to(torch.bfloat16).requires_grad_() for h in (HQ, HKV, HKV))
    cu = torch.tensor([0, 120, 300], dtype=torch.int32, device="cuda")
    f, factor = nsa.rotary_frequencies(128, scaling="parts", stretch=4.0)
    scores = torch.rand(T, HKV, 8, device="cuda")
    idx = nsa.select_blocks(scores, cu, 4)
    attn = nsa.SelAttention(T, HQ, HKV, 4, nseq=2)
    do = torch.randn(T, HQ, 128, device="cuda").to(torch.bfloat16)
    a, b = nsa.rotary(q, k, f, cu, factor=factor)
    o, _ = nsa.selected_attention(a, b, v, idx, attn, cu)
    o.backward(do)
    with torch.no_grad():
        a2, b2 = nsa.rotary(q, k, f, cu, factor=factor)
        o2, lse = attn.forward(a2, b2, v, idx, cu)
        da, db, dv = attn.backward(a2, b2, v, o2, lse, do, cu)
        dq, dk = nsa.rotary(da, db, -f, cu, factor=factor)
    assert torch.equal(o, o2) and torch.equal(v.grad, dv) and torch.equal(q.grad, dq) and torch.equal(k.grad, dk)


def test_empty():
    f, _ = nsa.rotary_frequencies()
    q = torch.zeros(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    assert nsa.rotary(q, None, f)[0].shape == (0, 4, 128)
    assert nsa.rotary(q, q, f, torch.zeros(4, dtype=torch.int32, device="cuda"))[1].shape == (0, 4, 128)
