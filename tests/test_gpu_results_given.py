"""Tensors that the calls write in place, as autograd sees them: a result that is given (and a page, a scale) has a new version after the call, so that a backward pass which saved
what was there refuses, as with torch's own operations in place, and does not take the new values for the old ones."""
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def _written(e4m3=False):
    """name -> (call, the tensors that it writes)."""
    cache = nsa.PagedCache(6, 2, page=64, dtype=E4M3 if e4m3 else BF)
    q, k = torch.randn(3, 8, 128, device="cuda").to(BF), torch.randn(3, 2, 128, device="cuda").to(BF)
    table, kv_len = torch.arange(6, dtype=I32, device="cuda").view(3, 2), torch.full((3,), 70, dtype=I32, device="cuda")
    f, _ = nsa.rotary_frequencies(64)
    scores = torch.rand(3, 2, 9, device="cuda")
    o, l, qo, ko, vo = torch.empty_like(q), torch.empty(3, 8, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
    idx = torch.empty(3, 2, 4, dtype=I32, device="cuda")
    pages = [x for x in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale) if x is not None]
    return {
        "rotary": (lambda: nsa.rotary(q, k, f, q_out=qo, k_out=ko), [qo, ko]),
        "rotary itself": (lambda: nsa.rotary(q, k, f, q_out=q, k_out=k), [q, k]),
        "rotary of q": (lambda: nsa.rotary(q, k, f, q_out=qo), [qo]),
        "append": (lambda: cache.append(k, k, table, kv_len, q=q, inv_freq=f, q_out=qo, k_out=ko), [qo, ko] + pages),
        "append of rows": (lambda: cache.append(k, k, table, kv_len), pages),
        "attention": (lambda: cache.attention(q, table, kv_len, out=o, lse=l), [o, l]),
        "attention_chunk": (lambda: cache.attention_chunk(q, table, kv_len, out=o, lse=l), [o, l]),
        "read": (lambda: cache.read(table, kv_len, k_out=ko, v_out=vo), [ko, vo]),
        "select_blocks": (lambda: nsa.select_blocks(scores, None, 4, kv_len=kv_len, out=idx), [idx]),
    }, [q, k, table, kv_len, f, scores, o, l, qo, ko, vo, idx, *pages]


NAMES = ["rotary", "rotary itself", "rotary of q", "append", "append of rows", "attention", "attention_chunk", "read", "select_blocks"]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_what_is_written_has_a_new_version(name, e4m3):
    calls, every = _written(e4m3)
    call, written = calls[name]
    before = [x._version for x in every]
    call()
    for x, v in zip(every, before):
        assert (x._version > v) == any(x is w for w in written), name


@pytest.mark.parametrize("name", NAMES)
def test_inference_tensors_are_written_as_before(name):
    """They have no version, inside inference mode and outside."""
    with torch.inference_mode():
        calls, _ = _written()
        calls[name][0]()
    calls[name][0]()


def test_a_backward_pass_does_not_take_what_was_written_for_what_it_saved():
    f, _ = nsa.rotary_frequencies(128)
    q = torch.randn(9, 4, 128, device="cuda").to(BF)
    w = torch.randn_like(q).requires_grad_()
    z = (q * w).sum()
    nsa.rotary(q, None, f, q_out=q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    base = torch.randn(9, 12, 128, device="cuda").to(BF)                     # a slice in place is a change of the whole
    z = (base * torch.randn_like(base).requires_grad_()).sum()
    nsa.rotary(base[:, :8], None, f, q_out=base[:, :8])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
