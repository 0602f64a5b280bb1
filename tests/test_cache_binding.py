"""What the Python calls over a paged cache look at in every call, on the host."""
import pytest
import torch

import paper_2508_18224_amd as nsa

F8 = torch.float8_e4m3fn
NAMES = ["k_pages", "v_pages", "k_scale", "v_scale"]


def _tensors(n_pages=5, dtype=F8):
    pages = [torch.zeros(n_pages, 2, 64, 128, dtype=dtype) for _ in range(2)]
    return pages + ([torch.ones(n_pages, 2) for _ in range(2)] if dtype is F8 else [])


def _calls(cache):
    i32, bf = torch.int32, torch.bfloat16
    q, k = torch.zeros(3, 8, 128, dtype=bf), torch.zeros(3, 2, 128, dtype=bf)
    table, kv_len = torch.zeros(3, 4, dtype=i32), torch.ones(3, dtype=i32)
    return [lambda: cache.append(k, k, table, kv_len, q=q), lambda: cache.attention(q, table, kv_len)]


def test_what_a_cache_is_made_of_cannot_be_replaced():
    """An attribute that could be assigned would be ignored by the calls."""
    cache = nsa.PagedCache.from_tensors(*_tensors())
    for name in NAMES + ["n_pages", "hkv", "page", "device"]:
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name))


@pytest.mark.parametrize("which", range(4))
def test_storage_that_is_gone_is_refused(which):
    """As where an engine gives a cache's memory back for a while; a tensor with an offset has an address that is not null then."""
    for offset in (0, 1):
        t = _tensors()
        whole = torch.stack([t[which]] * 2) if which >= 2 else torch.stack([t[which].view(torch.uint8)] * 2).view(F8)
        t[which] = whole[offset]
        cache = nsa.PagedCache.from_tensors(*t)
        for size in (0, whole.untyped_storage().nbytes() // 4):
            whole.untyped_storage().resize_(size)
            for call in _calls(cache):
                with pytest.raises(nsa.NsaSelError, match=NAMES[which]):
                    call()


@pytest.mark.parametrize("which", range(4))
def test_tensors_that_became_others_are_refused(which):
    cache = nsa.PagedCache.from_tensors(*_tensors())
    was, mine = _tensors()[which], getattr(cache, NAMES[which])
    others = [_tensors(6)[which], was.view(torch.int8) if which < 2 else was.half(), torch.stack([was.view(torch.int8)] * 2, -1)[..., 0].view(F8) if which < 2 else
              torch.stack([was] * 2, -1)[..., 0]]
    for other in others:
        mine.data = other
        for call in _calls(cache):
            with pytest.raises(nsa.NsaSelError, match=NAMES[which]):
                call()


def test_gradients_are_refused_not_lost():
    """Neither call has a backward: in grad mode a tensor that requires grad is refused, by its name; without grad mode it is a tensor like others."""
    bf, i32 = torch.bfloat16, torch.int32
    q, k, f = torch.zeros(3, 8, 128, dtype=bf), torch.zeros(3, 2, 128, dtype=bf), torch.zeros(64, dtype=torch.float64)
    gate, lse = torch.zeros(3, 8), torch.zeros(3, 8)
    table, kv_len = torch.zeros(3, 4, dtype=i32), torch.ones(3, dtype=i32)
    cache = nsa.PagedCache(5, 2, device="cpu")
    append = dict(k=k, v=k.clone(), q=q, inv_freq=f, q_out=q.clone(), k_out=k.clone())
    attention = dict(q=q, gate=gate, o_acc=q.clone(), out=q.clone(), lse=lse)
    for call, args in ((cache.append, append), (cache.attention, attention)):
        for name in args:
            mine = {**args, name: args[name].clone().requires_grad_()}
            with pytest.raises(nsa.NsaSelError, match=f"^{name} requires grad"):
                call(table=table, kv_len=kv_len, **mine)
            with torch.no_grad(), pytest.raises(nsa.NsaSelError, match="device tensors"):  # all that is wrong here
                call(table=table, kv_len=kv_len, **mine)
    cache.k_pages.requires_grad_()
    for call, args in ((cache.append, append), (cache.attention, attention)):
        with pytest.raises(nsa.NsaSelError, match="^k_pages requires grad"):
            call(table=table, kv_len=kv_len, **args)
    with pytest.raises(nsa.NsaSelError, match="device tensors"):                              # ids have no gradient to lose
        nsa.select_blocks(torch.zeros(3, 2, 8, requires_grad=True), None, 4, kv_len=kv_len)


def test_workspace_sizes_of_numbers_that_are_too_large():
    """They would be taken modulo 2^32: the size of another call."""
    cache = nsa.PagedCache(5, 2, device="cpu")
    ok = dict(tokens=3, hq=8, nseq=3, max_pages=4000, topk=0, block=64, window=0)
    assert cache.workspace_bytes(**ok) > 0
    for name in ok:
        for far in (2 ** 32, -2 ** 32, 2 ** 31):
            with pytest.raises(nsa.NsaSelError, match=f"^{name} is out of range"):
                cache.workspace_bytes(**{**ok, name: ok[name] + far if far != 2 ** 31 else far})
