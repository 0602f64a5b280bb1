"""The calls that are handed to the library past torch's dispatcher: what a transform of torch would lose without an error is refused.  On the host: the refusals come before any launch."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_2508_18224_amd as nsa

BF, I32 = torch.bfloat16, torch.int32


def _calls():
    """Each call as a function of one of its tensors, and that tensor."""
    cache = nsa.PagedCache(5, 2, page=64, device="cpu")
    q, k = torch.randn(3, 8, 128).to(BF), torch.randn(3, 2, 128).to(BF)
    table, kv_len = torch.zeros(3, 4, dtype=I32), torch.ones(3, dtype=I32)
    f, _ = nsa.rotary_frequencies(64, device="cpu")
    scores, gate = torch.rand(3, 2, 9), torch.rand(3, 8)
    return {
        "rotary": (lambda x: nsa.rotary(x, k, f), q),
        "rotary of k": (lambda x: nsa.rotary(q, x, f), k),
        "rotary's frequencies": (lambda x: nsa.rotary(q, k, x), f),
        "rotary in place": (lambda x: nsa.rotary(x, None, f, q_out=q.clone()), q),
        "append": (lambda x: cache.append(x, k, table, kv_len), k),
        "append of q": (lambda x: cache.append(k, k, table, kv_len, q=x, inv_freq=f), q),
        "attention": (lambda x: cache.attention(x, table, kv_len), q),
        "attention's gate": (lambda x: cache.attention(q, table, kv_len, gate=x), gate),
        "attention_chunk": (lambda x: cache.attention_chunk(x, table, kv_len), q),
        "attention_chunk's gate": (lambda x: cache.attention_chunk(q, table, kv_len, gate=x), gate),
        "read": (lambda x: cache.read(table, kv_len, k_out=x), k),
        "select_blocks": (lambda x: nsa.select_blocks(x, None, 4, kv_len=kv_len), scores),
    }


NAMES = list(_calls())


@pytest.mark.parametrize("name", NAMES)
def test_as_they_are(name):
    """(All that is wrong with the calls below.)"""
    call, x = _calls()[name]
    with pytest.raises(nsa.NsaSelError, match="device tensors"):
        call(x)


@pytest.mark.parametrize("grad", ["on", "off", "inference"])
@pytest.mark.parametrize("requires_grad", [False, True])
@pytest.mark.parametrize("name", [n for n in NAMES if n != "select_blocks"])
def test_a_forward_gradient_is_refused(name, requires_grad, grad):
    """Without grad mode too: forward gradients go on there, and only inference mode leaves them out."""
    call, x = _calls()[name]
    with fwd.dual_level():
        x = fwd.make_dual(x.clone().requires_grad_(requires_grad), torch.ones_like(x))
        if grad == "inference":
            with torch.inference_mode(), pytest.raises(nsa.NsaSelError, match="device tensors"):
                call(x)
        elif grad == "on":
            with pytest.raises(nsa.NsaSelError, match="forward|requires grad"):
                call(x)
        else:
            with torch.no_grad(), pytest.raises(nsa.NsaSelError, match="forward"):
                call(x)


def test_block_ids_have_no_forward_gradient():
    call, x = _calls()["select_blocks"]
    with fwd.dual_level(), pytest.raises(nsa.NsaSelError, match="device tensors"):
        call(fwd.make_dual(x, torch.ones_like(x)))


@pytest.mark.parametrize("name", NAMES)
def test_other_transforms_raise(name):
    call, x = _calls()[name]
    first = lambda x: call(x)[0] if name != "select_blocks" else call(x)  # noqa: E731
    for transformed in (lambda: torch.vmap(first)(torch.stack([x, x])), lambda: torch.func.jvp(first, (x,), (torch.ones_like(x),)),
                        lambda: torch.func.grad(lambda y: first(y).float().sum())(x), lambda: torch.func.functionalize(first)(x)):
        with pytest.raises(Exception):
            transformed()
