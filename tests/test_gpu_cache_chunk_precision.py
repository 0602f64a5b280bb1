"""What a row's probabilities are taken against in the attention of pieces: its true maximum so far, so that the largest one is 1, which bf16 holds exactly."""
import math

import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
def test_the_largest_probability_is_exact(e4m3):
    """Two keys weigh anything: one with a score of 0 and values of 0 in the first piece, then one with a score between 0 and 6 ln 2, a different one for every row, and values of 1.  The second has
    the largest probability, which is rounded for its product unless it is 1; the first one's meets a zero.  So O is exp(x) / (1 + exp(x)) but for 32-bit errors: x is a product of two bf16 values
    and the scale, 2^-23 of it each for the product, its factor log2(e) and the base-2 exponential's argument, whose own error and the quotient's are a few 2^-24: below 2^-19 in all, 2^-18 allowed.
    o_acc takes the result rounded to bf16 away, so that what is left is rounded below 2^-8 of 2^-8."""
    T, page, L = 256, 64, 64 * 6
    k, v = np.zeros((L // page, 1, page, 128)), np.zeros((L // page, 1, page, 128))
    k[..., 1] = -64.0                                                         # all others: -64 * 64 * scale
    k[0, 0, 3] = 0.0
    k[1, 0, 5] = 0.0
    k[1, 0, 5, 0], v[1, 0, 5] = 1.0, 1.0
    cache = nsa.PagedCache.from_tensors(*(dev(x, E4M3 if e4m3 else torch.bfloat16) for x in (k, v)), *([torch.ones(L // page, 1, device="cuda") for _ in range(2)] if e4m3 else []))
    scale = 0.125
    q = np.zeros((T, 1, 128))
    q[..., 1] = 64.0
    q[:, 0, 0] = np.arange(1, T + 1) / 256 * 6 * math.log(2) / scale
    q = host(dev(q, torch.bfloat16))
    x = q[:, 0, 0] * scale
    want = np.exp(x) / (1 + np.exp(x))
    near = host(dev(want, torch.bfloat16))
    acc = dev(-np.broadcast_to(near[:, None, None], (T, 1, 128)), torch.bfloat16)
    table = torch.arange(L // page, dtype=torch.int32, device="cuda")[None]
    kv_len, cu = dev(np.array([L + T]), torch.int32), dev(np.array([0, T]), torch.int32)
    o, _ = cache.attention_chunk(dev(q, torch.bfloat16), table, kv_len, cu, scale=scale, gate=torch.ones(T, 1, device="cuda"), o_acc=acc)
    left = (want - near)[:, None, None]
    assert (np.abs(host(o) - left) <= 2.0 ** -8 * np.abs(left) + 2.0 ** -18).all()


@pytest.mark.parametrize("spread", [1.0, 2.0, 4.0, 8.0])
def test_norm_of_the_error(spread):
    """2048 rows behind 8192 keys, scores of this spread: the norm of the error against that of a softmax in 64 bits whose probabilities are rounded to bf16 against the true maximum.  Both are
    norms of at least 2048 independent roundings' sums, whose squares scatter by 0.9 / sqrt(2048) = 2 %, so the norms by 1 %: 4 % are allowed.  (Against a maximum that lags, up to 2^6 behind, the
    norm is 5 to 22 % larger.)"""
    rng = np.random.default_rng([81, int(spread)])
    L, n, page = 8192, 256, 64
    k, v = (torch.from_numpy(rng.standard_normal((L // page, 1, page, 128))).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.from_numpy(spread * rng.standard_normal((n, 8, 128))).to(torch.bfloat16).cuda()
    table = torch.from_numpy(rng.permutation(L // page).astype(np.int32)).cuda()[None]
    o, _ = nsa.PagedCache.from_tensors(k, v).attention_chunk(q, table, dev(np.array([L]), torch.int32), dev(np.array([0, n]), torch.int32))
    k, v = (x[table[0].long()][:, 0].reshape(L, 128).double() for x in (k, v))
    x = (torch.matmul(q.double().view(-1, 128), k.T.contiguous()) / math.sqrt(128)).view(n, 8, L)
    at = torch.arange(L, device="cuda")
    x = x.masked_fill(at[None, None] > (L - n + torch.arange(n, device="cuda"))[:, None, None], -math.inf).view(-1, L)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    total = p.sum(-1, keepdim=True)
    want, rounded = (torch.matmul(y, v) / total for y in (p, p.to(torch.bfloat16).double()))
    by_rounding = (rounded.to(torch.bfloat16).double() - want).norm()
    assert float((o.view(-1, 128).double() - want).norm() / by_rounding) <= 1.04
