"""Rotary positions, the cache read back and the attention of pieces of prompts, used as a program uses them: together, captured, on other streams, from several threads, far out in
memory, over batches drawn by lot."""
import threading

import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, Batch, bf16, check_attention, dev, host
from chunk_util import attend_chunks, check_chunks
from oracle import paged_cache_oracle as pco
from test_gpu_cache_far import _far
from test_gpu_cache_read import _check as check_read
from test_gpu_cache_serving import _captured
from test_gpu_rotary import _close, _places, _turned

pytestmark = pytest.mark.gpu
HQ, HKV, TOPK = 8, 2, 4


def _held(cache):
    return ([host(cache.k_pages), host(cache.v_pages)], [None, None] if cache.k_scale is None else [host(cache.k_scale), host(cache.v_scale)])


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_prompt_in_pieces(e4m3):
    """Prompts come in pieces: each is rotated and appended, attends to all that is there and to a window, gated; then the keys are read back for the training path's selected
    attention.  Against 64 bits on what the cache holds."""
    page, pieces = 32, [[100, 64, 1], [0, 130, 40], [77, 3, 200], [1, 1, 1]]
    n, most = 3, 300
    rng = np.random.default_rng(31)
    per = -(-most // page)
    table_h = rng.permutation(n * per).reshape(n, per).astype(np.int32)
    cache = nsa.PagedCache(n * per, HKV, page=page, dtype=E4M3 if e4m3 else torch.bfloat16)
    table = dev(table_h, torch.int32)
    f, _ = nsa.rotary_frequencies(128, device="cuda")
    have, rotated = np.zeros(n, dtype=np.int32), [[] for _ in range(n)]
    for new in pieces:
        T = sum(new)
        cu_h = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        places = np.concatenate([np.arange(h, h + c) for h, c in zip(have, new)]).astype(np.int32)
        have += np.array(new, dtype=np.int32)
        cu, kv_len = dev(cu_h, torch.int32), dev(have, torch.int32)
        q, k, v = (dev(rng.standard_normal((T, h, 128)), torch.bfloat16) for h in (HQ, HKV, HKV))
        # the same rotation by itself, the places given, and by the append
        rq, rk = nsa.rotary(q, k, f, positions=dev(places, torch.int32))
        aq, ak = cache.append(k, v, table, kv_len, cu, q=q, inv_freq=f, rotated_k=True)
        assert torch.equal(rq, aq) and torch.equal(rk, ak)
        gate = torch.rand(T, HQ, device="cuda")
        everything, lse = cache.attention_chunk(rq, table, kv_len, cu)
        both, window_lse = cache.attention_chunk(rq, table, kv_len, cu, window=50, gate=gate, o_acc=everything)
        pages, scales = _held(cache)
        most_v = np.nanmax(np.abs(pages[1])) * (1.0 if scales[1] is None else scales[1].max())
        check_chunks(everything, lse, attend_chunks(host(rq), table_h, have, cu_h, pages, scales, page), keys=most, most=most_v)
        check_chunks(both, window_lse, attend_chunks(host(rq), table_h, have, cu_h, pages, scales, page, window=50), host(gate), host(everything), keys=most, most=most_v)
        for s in range(n):
            rotated[s].append(rq[cu_h[s]:cu_h[s + 1]])
    # whole sequences out of the cache, for the training path
    total = int(have.sum())
    cu_h = np.concatenate([[0], np.cumsum(have)]).astype(np.int32)
    cu, kv_len = dev(cu_h, torch.int32), dev(have, torch.int32)
    k, v = cache.read(table, kv_len, cu, tokens=total)
    rq = torch.cat([x for s in rotated for x in s])
    idx = nsa.select_blocks(torch.rand(total, HKV, 8, device="cuda"), cu, TOPK)
    o, lse = nsa.SelAttention(total, HQ, HKV, TOPK, nseq=n, bwd=False).forward(rq, k, v, idx, cu)
    pages, scales = _held(cache)
    check_attention(o, lse, pco.attend(host(rq), table_h, have, cu_h, pages, scales, page, idx=idx.cpu().numpy(), block=64))


@pytest.mark.parametrize("e4m3", [False, True])
def test_captured_and_replayed(e4m3):
    """The three in one graph, replayed with other data and lengths and eager work between; units that many workgroups share and such as are whole."""
    kv = np.array([3000, 90, 700, 0], dtype=np.int32)
    b = Batch(151, kv + 8, [40, 1, 300, 8], hq=HQ, hkv=HKV, page=32, e4m3=e4m3)
    for x in b.pages:
        x[np.isnan(x)] = 0.0
    cache = b.upload(nsa)
    f, _ = nsa.rotary_frequencies(128, device="cuda")
    gate = torch.rand(b.T, HQ, device="cuda")

    def run():
        q, k = nsa.rotary(b.dq, b.dk, f, b.dcu)
        o, l = cache.attention_chunk(q, b.dtable, b.dlen, b.dcu)
        w, m = cache.attention_chunk(q, b.dtable, b.dlen, b.dcu, window=100, gate=gate, o_acc=o)
        x, y = cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T)
        return q, k, o, l, w, m, x, y

    g, held = _captured(run)
    other = torch.randn(1 << 20, device="cuda")
    for i in range(5):
        b.dq.normal_()
        b.dk.normal_()
        b.dlen.copy_(dev(kv + 2 * i, torch.int32))
        eager = [x.clone() for x in run()]
        other.mul_(1.0001).sum().item()
        for x in held:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, eager):
            assert torch.equal(a, c)


def test_a_captured_backward_pass():
    """The rotation's forward and backward pass in a graph, replayed with other data and eager passes between; the leaves are made where the graph is."""
    q, k, gq, gk = (torch.randn(150, h, 128, device="cuda").to(torch.bfloat16) for h in (HQ, HKV, HQ, HKV))
    cu = dev(np.array([0, 70, 150], dtype=np.int32), torch.int32)
    f, factor = nsa.rotary_frequencies(64, scaling="parts", stretch=4.0, device="cuda")

    def run():
        a, b = q.detach().requires_grad_(), k.detach().requires_grad_()
        x, y = nsa.rotary(a, b, f, cu, factor=factor)
        return (x.detach(), y.detach(), *torch.autograd.grad((x, y), (a, b), (gq, gk)))

    g, held = _captured(run)
    for _ in range(4):
        for x in (q, k, gq, gk):
            x.normal_()
        eager = [x.clone() for x in run()]
        for x in held:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, eager):
            assert torch.equal(a, c)


def test_gradients_as_a_program_may_ask_for_them():
    """Twice of one pass; on a stream of its own; for one input; through a hook; not after the graph is gone or after the places were changed."""
    q, k, g = (torch.randn(90, h, 128, device="cuda").to(torch.bfloat16) for h in (HQ, HKV, HQ))
    places = torch.arange(90, dtype=torch.int32, device="cuda") * 3
    f, _ = nsa.rotary_frequencies(96, device="cuda")
    want = nsa.rotary(g, None, -f, positions=places)[0]
    a = q.clone().requires_grad_()
    x, y = nsa.rotary(a, k, f, positions=places)
    assert x.requires_grad and x.grad_fn is not None
    for _ in range(2):
        assert torch.equal(torch.autograd.grad(x, a, g, retain_graph=True)[0], want)
    seen = []
    x.register_hook(lambda grad: seen.append(grad) or 2 * grad)
    assert torch.equal(torch.autograd.grad(x, a, g)[0], nsa.rotary(2 * g, None, -f, positions=places)[0]) and torch.equal(seen[0], g)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(x, a, g)                                  # the graph is gone
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        b = q.detach().clone().requires_grad_()
        x, _ = nsa.rotary(b, k, f, positions=places)
        (d,) = torch.autograd.grad(x, b, g)
    assert not s.query()
    s.synchronize()
    assert torch.equal(d, want)
    with torch.no_grad():
        assert not nsa.rotary(a, k, f, positions=places)[0].requires_grad
    x, _ = nsa.rotary(a, k, f, positions=places)
    places.add_(1)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(x, a, g)                                  # the places of the pass are no longer there


def test_two_graphs_and_an_eager_call_at_once():
    """Workspaces of calls that run beside each other are apart."""
    batches = [Batch(160 + i, [3000 - 700 * i, 70, 1900], [50, 70, 33 + i], hq=HQ, hkv=HKV, page=64, e4m3=i == 1) for i in range(2)]
    graphs, held, want = [], [], []
    for b in batches:
        cache = b.upload(nsa)
        run = lambda b=b, cache=cache: (*cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu), *cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T))  # noqa: E731
        want.append([x.clone() for x in run()])
        g, h = _captured(run)
        graphs.append(g)
        held.append(h)
    streams = [torch.cuda.Stream() for _ in range(3)]
    a = batches[0]
    for _ in range(5):
        for h in held:
            for x in h:
                x.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            eager = (*a.cache.attention_chunk(a.dq, a.dtable, a.dlen, a.dcu), *a.cache.read(a.dtable, a.dlen, a.dcu, tokens=a.T))
        torch.cuda.synchronize()
        for got, w in zip(held + [eager], want + [want[0]]):
            assert all(torch.equal(x, y) for x, y in zip(got, w))


def test_calls_go_to_the_current_stream():
    b = Batch(162, [500, 90], [40, 90], hq=HQ, hkv=HKV, page=64)
    cache = b.upload(nsa)
    f, _ = nsa.rotary_frequencies(128, device="cuda")

    def run(q):
        x, y = nsa.rotary(q, b.dk, f, b.dcu)
        return (*cache.attention_chunk(x, b.dtable, b.dlen, b.dcu), *cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T), y)

    want = [x.clone() for x in run(b.dq)]
    q = torch.zeros_like(b.dq)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        q.copy_(b.dq)
        got = run(q)
    assert not s.query()
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_calls_of_several_threads():
    batches = [Batch(163 + i, [900 - 100 * i, 70 + i, 300], [30, 70, 150], hq=HQ, hkv=HKV, page=64, e4m3=i % 2 == 1) for i in range(4)]
    f, _ = nsa.rotary_frequencies(64, device="cuda")

    def step(b):
        leaf = b.dq.detach().requires_grad_()
        q, k = nsa.rotary(leaf, b.dk, f, b.dcu)
        (dq,) = torch.autograd.grad(q, leaf, b.dq)
        return (q.detach(), k.detach(), dq, *b.cache.attention_chunk(q.detach(), b.dtable, b.dlen, b.dcu, window=200), *b.cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T))

    want = []
    for b in batches:
        b.upload(nsa)
        want.append([x.clone() for x in step(b)])
    got, failed = [None] * 4, []
    torch.cuda.synchronize()

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(30):
                    got[i] = step(batches[i])
            s.synchronize()
        except Exception as e:  # shown by the assertion below
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for g, w in zip(got, want):
        assert all(torch.equal(a, c) for a, c in zip(g, w))


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_past_four_gigabytes(e4m3):
    """What lies at the far end of a large cache is read and attended to as at the near end of a small one."""
    b = Batch(170, [300, 5000, 33], [150, 90, 33], hq=8, hkv=4, page=64, e4m3=e4m3)
    near = b.upload(nsa)
    far, table = _far(near, b)
    for run in (lambda c, t: c.attention_chunk(b.dq, t, b.dlen, b.dcu), lambda c, t: c.attention_chunk(b.dq, t, b.dlen, b.dcu, window=70),
                lambda c, t: c.read(t, b.dlen, b.dcu, tokens=b.T)):
        want, got = run(near, b.dtable), run(far, table)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_that_lie_far_apart():
    """Tokens more than 2^31 values apart: of the rotation's arguments and results, and of what is read into."""
    b = Batch(171, [70, 3, 64], [1, 1, 1], hq=8, hkv=4, page=64)
    cache = b.upload(nsa)
    f, _ = nsa.rotary_frequencies(128, device="cuda")
    stride = 2 ** 30 + 2 ** 11
    whole = torch.empty(2 * stride + 20 * 128, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(whole, (3, 20, 128), (stride, 128, 1))
    rows[:, :8], rows[:, 8:12] = b.dq, b.dk
    places = dev(np.array([5, 1000, 70000], dtype=np.int32), torch.int32)
    want = nsa.rotary(b.dq, b.dk, f, positions=places)
    nsa.rotary(rows[:, :8], rows[:, 8:12], f, positions=places, q_out=rows[:, :8], k_out=rows[:, 8:12])
    assert torch.equal(rows[:, :8], want[0]) and torch.equal(rows[:, 8:12], want[1])
    want = cache.read(b.dtable, b.dlen)
    cache.read(b.dtable, b.dlen, k_out=rows[:, 12:16], v_out=rows[:, 16:])
    assert torch.equal(rows[:, 12:16], want[0]) and torch.equal(rows[:, 16:], want[1])


@pytest.mark.parametrize("n", [9, 300])
@pytest.mark.parametrize("e4m3", [False, True])
def test_idle_slots(n, e4m3):
    """Sequences whose one new token has a negative place: their rows are zero and what their queries hold does not matter."""
    lens = np.where(np.arange(n) % 3 == 1, 0, 1 + 7 * (np.arange(n) % 40))
    lens[4] = -3
    b = Batch(172, lens, hq=8, hkv=2, page=32, e4m3=e4m3)
    b.q[lens <= 0] = np.nan
    cache = b.upload(nsa)
    o, lse = cache.attention_chunk(b.dq, b.dtable, b.dlen)
    check_chunks(o, lse, attend_chunks(np.nan_to_num(b.q), b.table, b.kv_len, None, b.pages, b.scales, 32), keys=300, most=448.0)
    off = torch.from_numpy(lens <= 0).cuda()
    assert (o[off] == 0).all() and torch.isneginf(lse[off]).all()
    k, v = cache.read(b.dtable, b.dlen)
    assert (k[off] == 0).all() and (v[off] == 0).all()


def test_largest_values():
    """Values of the largest size that bf16 holds: a key in 64 has all the weight, each five times as much in powers of two as the one before it and with the other sign, so that the
    results are finite, and stay so wherever the running sums are rescaled."""
    most = float(torch.finfo(torch.bfloat16).max)
    b = Batch(173, [700, 90], [64, 90], hq=8, hkv=2, page=64)
    for s in range(2):
        for u in range(int(b.kv_len[s])):
            p = b.table[s, u // 64]
            b.pages[0][p, :, u % 64] = bf16(np.full(128, 5 * np.log(2) / 128 * (u // 64) if u % 64 == 10 else -3.0))
            b.pages[1][p, :, u % 64] = most * (-1) ** (u // 64)
    b.q = bf16(np.full(b.q.shape, 1.0))
    cache = b.upload(nsa)
    o, lse = cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, scale=1.0)
    assert torch.isfinite(lse).all()
    seen = slice(64 + 10, None)  # the first tokens of the second sequence see keys of equal score, whose sum is beyond 32 bits
    assert torch.isfinite(o[:64].float()).all() and torch.isfinite(o[seen].float()).all()
    ref = attend_chunks(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, 64, scale=1.0)
    for rows in (slice(0, 64), seen):
        check_chunks(o[rows], lse[rows], tuple(x[rows] for x in ref), keys=700, most=most)


def test_lengths_of_any_sign():
    """The least length that a number of 32 bits holds is a negative one like others: nothing is seen, rows are zero."""
    b = Batch(175, [70, 300, 40], hq=8, hkv=2, page=32)
    cache = b.upload(nsa)
    b.dlen[0], b.dlen[2] = -2 ** 31, -2 ** 31 + 5
    o, lse = cache.attention_chunk(b.dq, b.dtable, b.dlen)
    k, v = cache.read(b.dtable, b.dlen)
    for i in (0, 2):
        assert (o[i] == 0).all() and torch.isneginf(lse[i]).all() and (k[i] == 0).all() and (v[i] == 0).all()
    assert torch.isfinite(lse[1]).all() and (k[1] != 0).any()
    far = torch.full_like(b.dlen, 2 ** 31 - 1)                           # past the table: what it holds is seen, a place without a page is zero
    o, lse = cache.attention_chunk(b.dq, b.dtable, far, window=5)
    assert (o == 0).all() and torch.isneginf(lse).all()
    assert (cache.read(b.dtable, far)[0] == 0).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_results_in_place_of_the_sum_so_far(e4m3):
    """out may be o_acc: units that one workgroup has, and such as are joined from parts."""
    b = Batch(174, [5000, 300, 64], [40, 130, 64], hq=8, hkv=2, page=32, e4m3=e4m3)
    cache = b.upload(nsa)
    gate = torch.rand(b.T, 8, device="cuda")
    acc = torch.randn(b.T, 8, 128, device="cuda").to(torch.bfloat16)
    for window in (0, 90):
        want, lse = cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, window=window, gate=gate, o_acc=acc)
        both = acc.clone()
        got = cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, window=window, gate=gate, o_acc=both, out=both)
        assert got[0] is both and torch.equal(both, want) and torch.equal(got[1], lse)


@pytest.mark.parametrize("seed", range(24))
def test_drawn_by_lot(seed):
    """Heads, pages, lengths, windows, gates, both formats, rotations of every kind."""
    rng = np.random.default_rng([181, seed])
    hkv, g = int(rng.choice([1, 2, 3, 4])), int(rng.choice([1, 2, 3, 4, 7, 8]))
    hq, page, n = hkv * g, int(rng.choice([16, 32, 64, 128, 256])), int(rng.integers(1, 6))
    new = [int(x) for x in rng.choice([0, 1, 2, 17, 63, 64, 65, 130, 257], n)]
    kv = [c + int(x) for c, x in zip(new, rng.choice([0, 1, 63, 64, 500, 1500], n))]
    b = Batch(1000 + seed, kv, new, hq=hq, hkv=hkv, page=page, e4m3=bool(seed % 2), pad=int(rng.integers(0, 3)), before=int(rng.integers(0, 3)))
    cache = b.upload(nsa)
    window = int(rng.choice([0, 1, 64, 200]))
    gated = bool(rng.integers(0, 2))
    gate = rng.standard_normal((b.T, hq)).astype(np.float32) if gated else None
    acc = bf16(rng.standard_normal((b.T, hq, 128))) if gated else None
    if b.T:
        o, lse = cache.attention_chunk(b.dq, b.dtable, b.dlen, b.dcu, window=window, gate=dev(gate, torch.float32), o_acc=dev(acc, torch.bfloat16))
        ref = attend_chunks(b.q, b.table, b.kv_len, b.cu, b.pages, b.scales, page, window=window)
        most = np.nanmax(np.abs(b.pages[1]), initial=0.0) * (1.0 if b.scales[1] is None else b.scales[1].max())
        check_chunks(o, lse, ref, None if gate is None else gate.astype(np.float64), acc, keys=max(kv), most=most)
        check_read(b, *cache.read(b.dtable, b.dlen, b.dcu, tokens=b.T), None)
    rot, interleaved, factor = int(rng.choice([16, 48, 64, 128])), bool(rng.integers(0, 2)), float(rng.choice([1.0, 0.7, 1.3]))
    f = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    x, y = nsa.rotary(b.dq, b.dk, dev(f, torch.float64), b.dcu, interleaved=interleaved, factor=factor)
    _close(x, _turned(b.q, _places([int(c) for c in b.cu], b.T), f, interleaved, factor))
    _close(y, _turned(b.k, _places([int(c) for c in b.cu], b.T), f, interleaved, factor))
