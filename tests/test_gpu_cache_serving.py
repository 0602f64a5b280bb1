"""The cache calls together, as a model that serves uses them: a prompt, tokens one by one, drafts; captured, on other streams, two at once."""
import numpy as np
import pytest
import torch

import paper_2508_18224_amd as nsa
from cache_util import E4M3, Batch, bf16, check_attention, dev, host
from oracle import paged_cache_oracle as pco

pytestmark = pytest.mark.gpu
HQ, HKV, TOPK, BLOCK = 8, 2, 4, 64


def _model(seed, lens, more):
    """Unrotated q, k, v of whole sequences, bf16 values."""
    rng = np.random.default_rng([23, seed])
    return [tuple(bf16(rng.standard_normal((L + more, h, 128))) for h in (HQ, HKV, HKV)) for L in lens]


@pytest.mark.parametrize("e4m3", [False, True])
def test_prompt_then_tokens_then_drafts(e4m3):
    """The prompt's keys go into the cache and, rotated, through the training path's forward; then 5 tokens one at a time and 4 at once, selected by
    scores over the cache.  Every attention is held to the oracle on what the cache holds, and what it holds to the oracle's append."""
    lens, page = [150, 33, 200], 16 if e4m3 else 64
    seqs = _model(1, lens, 9)
    n = len(lens)
    f = 10000.0 ** (-np.arange(0, 128, 2) / 128)
    df = dev(f, torch.float64)
    per = -(-(max(lens) + 9) // page)
    cache = nsa.PagedCache(n * per + 1, HKV, page=page, dtype=E4M3 if e4m3 else torch.bfloat16)
    table_h = np.random.default_rng(2).permutation(n * per).reshape(n, per).astype(np.int32)
    table = dev(table_h, torch.int32)
    shape = (n * per + 1, HKV, page, 128)
    pages = [np.zeros(shape), np.zeros(shape)]
    scales = [np.ones(shape[:2]), np.ones(shape[:2])] if e4m3 else [None, None]
    have = [0] * n

    def step(counts, name):
        """Appends `counts` tokens of each sequence, attends, checks; returns the rotated queries and keys."""
        kv = np.array([h + c for h, c in zip(have, counts)], dtype=np.int32)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        q, k, v = (np.concatenate([s[i][h:h + c] for s, h, c in zip(seqs, have, counts)]) for i in range(3))
        one = all(c == 1 for c in counts)
        dcu = None if one else dev(cu, torch.int32)
        dlen = dev(kv, torch.int32)
        rq, rk = cache.append(dev(k, torch.bfloat16), dev(v, torch.bfloat16), table, dlen, dcu, q=dev(q, torch.bfloat16), inv_freq=df, rotated_k=True)
        pco.append(k, v, table_h, kv, cu, pages, scales, page, f)
        for x, ref, s in ((cache.k_pages, pages[0], scales[0]), (cache.v_pages, pages[1], scales[1])):
            err = np.abs(host(x) - ref)                    # an angle's error may put a value on the other side of a border: one step of the format
            assert (err <= np.abs(ref) * (2.0 ** -3 if e4m3 else 2.0 ** -7) + (2.0 ** -9 if e4m3 else 0)).all()
            assert (err > 0).mean() < 1e-2
        stride = -(-int(kv.max()) // BLOCK)
        x = np.random.default_rng([3, int(kv[0])]).standard_normal((len(q), HKV, stride)).astype(np.float32)
        idx = nsa.select_blocks(dev(x, torch.float32), dcu, TOPK, kv_len=dlen)
        idx_ref = pco.select(x, kv, None if one else cu, TOPK)
        assert np.array_equal(idx.cpu().numpy(), idx_ref), name
        o, lse = cache.attention(rq, table, dlen, dcu, idx=idx, block=BLOCK)
        held = [host(cache.k_pages), host(cache.v_pages)], [None, None] if not e4m3 else [host(cache.k_scale), host(cache.v_scale)]
        check_attention(o, lse, pco.attend(host(rq), table_h, kv, None if one else cu, held[0], held[1], page, idx=idx_ref, block=BLOCK))
        w, wl = cache.attention(rq, table, dlen, dcu, window=64)
        check_attention(w, wl, pco.attend(host(rq), table_h, kv, None if one else cu, held[0], held[1], page, window=64))
        for i, c in enumerate(counts):
            have[i] += c
        return rq, rk, idx, o, lse, dcu

    rq, rk, idx, o, lse, cu = step(lens, "prompt")
    if not e4m3:                                             # the training path's forward on the same rotated rows
        T = sum(lens)
        attn = nsa.SelAttention(T, HQ, HKV, TOPK, nseq=n, bwd=False)
        v = dev(np.concatenate([s[2][:L] for s, L in zip(seqs, lens)]), torch.bfloat16)
        o2, lse2 = attn.forward(rq, rk, v, idx, cu)
        # both are within their own rounding of the same value: 2^-8 of sum(p |v|) <= max |v| and of O, each
        most = float(v.float().abs().max())
        assert float((o.float() - o2.float()).abs().max()) <= 4 * 2.0 ** -8 * most
        assert float((lse - lse2).abs().max()) < 2e-3
    for i in range(5):
        step([1] * n, "token %d" % i)
    step([4, 0, 4], "drafts")


def _captured(run):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = run()
    return g, held


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("long", [False, True])
def test_a_step_is_captured_and_replayed(e4m3, long):
    """Append, selection, selected attention and attention to every key in one graph, replayed with other data, other lengths and eager work between."""
    kv = np.array([700, 90, 2000 if long else 300, 64], dtype=np.int32)
    b = Batch(51, kv + 8, hq=HQ, hkv=HKV, page=32, e4m3=e4m3)
    for x in b.pages:
        x[np.isnan(x)] = 0.0
    cache = b.upload(nsa)
    b.dlen.copy_(dev(kv + 1, torch.int32))
    f = dev(10000.0 ** (-np.arange(0, 128, 2) / 128), torch.float64)
    stride = int(kv.max() + 8) // 64 + 1
    scores = torch.rand(4, HKV, stride, device="cuda")
    start = [x.view(torch.uint8).clone() for x in (cache.k_pages, cache.v_pages)] + [None if x is None else x.clone() for x in (cache.k_scale, cache.v_scale)]

    def restore():
        cache.k_pages.view(torch.uint8).copy_(start[0])
        cache.v_pages.view(torch.uint8).copy_(start[1])
        if e4m3:
            cache.k_scale.copy_(start[2])
            cache.v_scale.copy_(start[3])

    def run():
        q, _ = cache.append(b.dk, b.dv, b.dtable, b.dlen, q=b.dq, inv_freq=f)
        idx = nsa.select_blocks(scores, None, TOPK, kv_len=b.dlen)
        o, l = cache.attention(q, b.dtable, b.dlen, idx=idx)
        w, m = cache.attention(q, b.dtable, b.dlen)
        return q, idx, o, l, w, m

    g, held = _captured(run)
    other = torch.randn(1 << 20, device="cuda")
    for i in range(4):
        b.dq.normal_()
        b.dk.normal_()
        b.dv.normal_()
        scores.uniform_()
        b.dlen.copy_(dev(kv + 1 + i, torch.int32))
        restore()
        eager = [x.clone() for x in run()]
        now = [x.view(torch.uint8).clone() for x in (cache.k_pages, cache.v_pages)]
        other.mul_(1.0001).sum().item()
        restore()
        for x in held:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, eager):
            assert torch.equal(a, c)
        assert torch.equal(cache.k_pages.view(torch.uint8), now[0]) and torch.equal(cache.v_pages.view(torch.uint8), now[1])


def test_two_graphs_and_two_streams_at_once():
    """Two captured calls that are replayed on two streams at once, and eager ones beside them, do not touch each other's workspaces."""
    a, b = (Batch(60 + i, [3000 - 500 * i, 70, 1900], hq=HQ, hkv=HKV, page=64) for i in range(2))
    graphs, held, want = [], [], []
    for x in (a, b):
        cache = x.upload(nsa)
        run = lambda x=x, cache=cache: cache.attention(x.dq, x.dtable, x.dlen)
        want.append([y.clone() for y in run()])
        g, h = _captured(run)
        graphs.append(g)
        held.append(h)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(10):
        for h in held:
            for y in h:
                y.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            eager = a.cache.attention(a.dq, a.dtable, a.dlen)
        torch.cuda.synchronize()
        for h, w in zip(held + [eager], want + [want[0]]):
            assert torch.equal(h[0], w[0]) and torch.equal(h[1], w[1])


def test_calls_go_to_the_current_stream():
    """A call waits for what its stream was given before, and nothing else."""
    b = Batch(62, [500, 40], hq=HQ, hkv=HKV, page=64)
    cache = b.upload(nsa)
    want = cache.attention(b.dq, b.dtable, b.dlen)[0].clone()
    q = torch.zeros_like(b.dq)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        q.copy_(b.dq)
        o, _ = cache.attention(q, b.dtable, b.dlen)
    assert not s.query()
    s.synchronize()
    assert torch.equal(o, want)


def test_calls_of_several_threads():
    """Threads with a stream each make all three calls at once, into caches of their own; each gets what it gets alone."""
    import threading
    batches = [Batch(63 + i, [900 - 100 * i, 70 + i, 300], hq=HQ, hkv=HKV, page=64, e4m3=i % 2 == 1) for i in range(4)]
    freq = dev(10000.0 ** (-np.arange(0, 128, 2) / 128), torch.float64)
    scores = [torch.rand(b.T, HKV, 16, device="cuda") for b in batches]

    def step(b, x):
        q, k = b.cache.append(b.dk, b.dv, b.dtable, b.dlen, q=b.dq, inv_freq=freq, rotated_k=True)
        idx = nsa.select_blocks(x, None, TOPK, kv_len=b.dlen)
        return (q, k, idx, *b.cache.attention(q, b.dtable, b.dlen, idx=idx), *b.cache.attention(q, b.dtable, b.dlen))

    want = []
    for b, x in zip(batches, scores):
        b.upload(nsa)
        step(b, x)  # appended again, a page's scale has grown already
        want.append([y.clone() for y in step(b, x)])
    got, failed = [None] * 4, []
    torch.cuda.synchronize()

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(50):
                    got[i] = step(batches[i], scores[i])
            s.synchronize()
        except Exception as e:  # shown by the assertion below
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))
