"""Positions, prompts in pieces over a paged cache, and the cache read back: three operators in plain form and through the library's calls.

A case is a dict of plain values:
  op        "rotary"  queries and keys of packed sequences turned by their places; with grad also the gradients of a training step
            "read"    keys and values of cached sequences as plain rows in bf16
            "chunk"   attention of a piece of a prompt over the cache that it has been appended to: of every key, or of a window
  seqs, shortest, longest   sequences of the batch and their lengths, the new tokens included (spread evenly over the logarithm); rotary and
            read take all tokens of a sequence
  new_least, new_most       new tokens of a sequence (chunk)
  hq, hkv, page, bits       heads, tokens per page, 16 (bf16) or 8 (e4m3 with a power-of-two scale for every page and head)
  rot, interleaved          rotated channels and how they pair
  far, stretch              the first place if places are given as a tensor (0: counted from the start of a sequence), and by how much
            the lower frequencies are stretched for contexts longer than the model was made for (1: not)
  sliced    queries and keys are slices of one projection
  window, gated             the window of the attention, and whether it adds into the gated sum of the branches

What the cache means: pages [n_pages, hkv, page, 128]; table [seqs, max_pages] names the page of every `page` tokens; kv_len holds
the lengths after the new tokens; new token i of n of a sequence has place kv_len - n + i.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
DEV = "cuda:0"
THETA = 500000.0


def _case(name, op, seqs, shortest, longest, hq, hkv, *, new_least=0, new_most=0, page=64, bits=16, rot=128, interleaved=False, far=0,
          stretch=1, sliced=False, grad=False, window=0, gated=False):
    c = dict(op=op, seqs=seqs, shortest=shortest, longest=longest, new_least=new_least, new_most=new_most, hq=hq, hkv=hkv, page=page,
             bits=bits, rot=rot, interleaved=interleaved, far=far, stretch=stretch, sliced=sliced, grad=grad, window=window, gated=gated)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token far out in a stretched context: what a call costs when there is nothing to move
        _case("rotary_1", "rotary", 1, 1, 1, 32, 8, far=900000, stretch=8),
        # a packed batch of odd lengths, Qwen-shaped heads, half of the channels, pairs side by side, slices of one projection; a training step
        _case("rotary_packed_grad", "rotary", 7, 333, 4001, 28, 4, rot=64, interleaved=True, sliced=True, grad=True),
        # the training step of a whole context of 64K tokens
        _case("rotary_64k_grad", "rotary", 1, 65536, 65536, 32, 8, grad=True),
        # a short conversation out of small pages
        _case("read_1", "read", 1, 513, 513, 8, 2, page=16),
        # the prefixes of a batch of prompts, 8 bits
        _case("read_64_e4m3", "read", 64, 100, 8000, 32, 8, bits=8),
        # one document of 128K tokens
        _case("read_128k", "read", 1, 131072, 131072, 32, 8),
        # a short question to a cached context: few rows, latency counts
        _case("chunk_16", "chunk", 1, 4096, 4096, 32, 8, new_least=16, new_most=16),
        # the usual piece of a long prompt
        _case("chunk_2048", "chunk", 1, 34816, 34816, 32, 8, new_least=2048, new_most=2048),
        # pieces of several prompts at once, uneven, Qwen-shaped heads, 8 bits
        _case("chunk_pieces_e4m3", "chunk", 7, 2333, 9001, 28, 4, new_least=333, new_most=2300, page=128, bits=8),
        # a whole prompt in one piece: nothing cached before it
        _case("chunk_whole_8k", "chunk", 1, 8192, 8192, 64, 8, new_least=8192, new_most=8192),
        # a short piece at the end of a very long document, 8 bits: one axis to split
        _case("chunk_512_long_e4m3", "chunk", 1, 131072, 131072, 64, 8, new_least=512, new_most=512, bits=8),
        # the sliding-window branch of a long piece, small pages, into the gated sum of the branches
        _case("chunk_window", "chunk", 1, 20000, 20000, 28, 4, new_least=8192, new_most=8192, page=16, window=512, gated=True),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "read", "chunk", "chunk", "chunk"])
    hq, hkv = rng.choice([(32, 8), (28, 4), (64, 8), (8, 8), (8, 2), (16, 2), (10, 2)])
    if op == "rotary":
        seqs = _between(rng, 1, 64)
        longest = _between(rng, 1, 60000 // seqs)
        return _case(None, op, seqs, _between(rng, 1, longest), longest, min(hq, 32), hkv, rot=rng.choice([16, 32, 64, 96, 128, 128, 128]),
                     interleaved=rng.random() < 0.4, far=rng.choice([0, 0, rng.randint(1, 1000000)]), stretch=rng.choice([1, 1, 4, 32]),
                     sliced=rng.random() < 0.4, grad=rng.random() < 0.6)
    page, bits = rng.choice([16, 32, 64, 128, 256]), rng.choice([8, 16])
    if op == "read":
        seqs = _between(rng, 1, 200)
        longest = _between(rng, 1, 130000 // seqs)
        return _case(None, op, seqs, _between(rng, 1, longest), longest, hq, hkv, page=page, bits=bits)
    seqs, most = _between(rng, 1, 12), _between(rng, 1, 4000)
    longest = most + _between(rng, 1, 60000)
    while seqs * hq * most * longest > 3 << 30:
        if seqs > 1:
            seqs -= 1
        else:
            longest = most + (longest - most) // 2
            most = min(most, 2000)
    shortest = most + _between(rng, 1, longest - most)
    return _case(None, op, seqs, shortest, longest, hq, hkv, new_least=_between(rng, 1, most), new_most=most, page=page, bits=bits,
                 window=rng.choice([0, 0, 0, _between(rng, 1, 4096)]), gated=rng.random() < 0.3)


# ---- sizes that follow from a case --------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    if n == 1:
        return [hi]
    return [max(lo, min(hi, int(round(lo * (hi / lo) ** (i / (n - 1)))))) for i in range(n)]


def _lengths(c):
    """(length, new tokens) of every sequence; neighbours are not neighbours in length."""
    n = c["seqs"]
    kv = _spread(n, c["shortest"], c["longest"])
    kv = [kv[(i * 5 + 3) % n] if math.gcd(5, n) == 1 else kv[i] for i in range(n)]
    return kv, _spread(n, c["new_least"], c["new_most"]) if c["op"] == "chunk" else list(kv)


def work(case):
    c = case
    kv, new = _lengths(c)
    T, size = sum(new), c["bits"] // 8
    if c["op"] == "rotary":
        passes = 2 if c["grad"] else 1
        return {"bytes": passes * T * (c["hq"] + c["hkv"]) * D * 2 * 2, "flops": passes * 3 * T * c["rot"] * (c["hq"] + c["hkv"])}
    if c["op"] == "read":
        return {"bytes": T * c["hkv"] * 2 * D * (size + 2), "flops": 0}
    w = c["window"]
    keys = 0
    for L, n in zip(kv, new):
        first = L - n + 1                                  # what the first new token sees without a window
        keys += n * first + n * (n - 1) // 2
        if w:
            over = max(0, L - w)                             # tokens that see more than the window: the last `over`, by 1 .. over
            fewer = max(0, over - n)
            keys -= over * (over + 1) // 2 - fewer * (fewer + 1) // 2
    reads = sum(min(L, w + n - 1) if w else L for L, n in zip(kv, new))
    moved = reads * c["hkv"] * 2 * D * size + T * c["hq"] * (2 * 2 * D + 4)
    if c["gated"]:
        moved += T * c["hq"] * (2 * D + 4)
    return {"bytes": moved, "flops": 4 * keys * c["hq"] * D}


# ---- inputs -----------------------------------------------------------------------------------------------------------------
def _pages(c, n_pages, gen, gain):
    x = torch.empty(n_pages, c["hkv"], c["page"], D, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    x *= gain
    if c["bits"] == 16:
        return x, None
    # the least power of two whose 448-fold holds the page
    most, s = x.float().abs().amax((2, 3)), torch.empty(n_pages, c["hkv"], device=DEV)
    s.copy_(torch.exp2(torch.ceil(torch.log2(most / 448.0))))
    out = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=DEV)
    for i in range(0, n_pages, 4096):
        out[i:i + 4096] = (x[i:i + 4096].float() / s[i:i + 4096, :, None, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return out, s


def _frequencies(c):
    """Radians per place, and what the turned channels are multiplied by: stretched contexts divide the frequencies that turn less
    than once in 8192 places, keep those that turn more than 32 times, and go over from one to the other in between."""
    f = THETA ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / c["rot"])
    if c["stretch"] == 1:
        return f, 1.0
    keep = ((8192 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return f * keep + f / c["stretch"] * (1 - keep), 0.1 * math.log(c["stretch"]) + 1


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kv, new = _lengths(c)
    T, n = sum(new), c["seqs"]
    st = {"c": c, "tokens": T, "longest": max(kv), "most": max(new)}
    starts = [0]
    for x in new:
        starts.append(starts[-1] + x)
    ints = dict(dtype=torch.int32, device=DEV)
    st["kv_len"], st["cu"] = torch.tensor(kv, **ints), torch.tensor(starts, **ints)

    def rows(heads):
        return torch.randn(T, heads, D, generator=gen, device=DEV).to(torch.bfloat16)

    # keys have a few strong channels, heads differ in size
    gain = torch.rand(1, c["hkv"], 1, 1, generator=gen, device=DEV) + 0.5
    strong = 1 + 3 * (torch.arange(D, device=DEV) % 32 == 5)
    if c["op"] == "rotary":
        q, k = rows(c["hq"]), (rows(c["hkv"]) * (gain[0, :, 0] * strong)).to(torch.bfloat16)
        if c["sliced"]:
            x = torch.cat((q, k, rows(c["hkv"])), 1)
            q, k = x[:, :c["hq"]], x[:, c["hq"]:c["hq"] + c["hkv"]]
        if c["grad"]:
            q, k = q.requires_grad_(), k.requires_grad_()
            st["gq"], st["gk"] = rows(c["hq"]), rows(c["hkv"])
        st["q"], st["k"] = q, k
        st["inv_freq"], st["factor"] = _frequencies(c)
        st["places"] = None
        if c["far"]:
            st["places"] = torch.cat([torch.arange(c["far"], c["far"] + x, **ints) for x in new])
        return st
    need = [(L + c["page"] - 1) // c["page"] for L in kv]
    n_pages = sum(need) + 5
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    width = max(need) + 2
    at = torch.arange(width, device=DEV)[None]
    have = torch.tensor(need, device=DEV)[:, None]
    first = torch.tensor([sum(need[:i]) for i in range(n)], device=DEV)[:, None]
    st["table"] = torch.where(at < have, order[(first + at).clamp(max=n_pages - 1)], -1).to(torch.int32)
    st["k_pages"], st["k_scale"] = _pages(c, n_pages, gen, (gain * strong).to(torch.bfloat16))
    st["v_pages"], st["v_scale"] = _pages(c, n_pages, gen, gain.to(torch.bfloat16))
    if c["op"] == "chunk":
        st["q"] = rows(c["hq"])
        if c["gated"]:
            st["gate"] = torch.rand(T, c["hq"], generator=gen, device=DEV)
            st["o_acc"] = rows(c["hq"])
    if own:
        import paper_2508_18224_amd as nsa
        st["cache"] = nsa.PagedCache.from_tensors(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(st):
    c = st["c"]
    if not own:
        return {"rotary": _rotary, "read": _read, "chunk": _chunk}[c["op"]](st)
    if c["op"] == "rotary":
        import paper_2508_18224_amd as nsa
        q, k = nsa.rotary(st["q"], st["k"], st["inv_freq"], st["cu"], positions=st["places"], interleaved=c["interleaved"], factor=st["factor"])
        if not c["grad"]:
            return q, k
        dq, dk = torch.autograd.grad((q, k), (st["q"], st["k"]), (st["gq"], st["gk"]))
        return q.detach(), k.detach(), dq, dk
    if c["op"] == "read":
        return st["cache"].read(st["table"], st["kv_len"], st["cu"], tokens=st["tokens"])
    return st["cache"].attention_chunk(st["q"], st["table"], st["kv_len"], st["cu"], window=c["window"], gate=st.get("gate"), o_acc=st.get("o_acc"))


def _where(st):
    """Sequence, number in it and place of every token."""
    kv, cu = st["kv_len"].long(), st["cu"].long()
    t = torch.arange(st["tokens"], device=DEV)
    s = torch.searchsorted(cu, t, right=True) - 1
    i = t - cu[s]
    return s, i, kv[s] - (cu[s + 1] - cu[s]) + i


def _turned(x, co, si, interleaved):
    """x with its first channels turned by the angles whose cosine and sine are given; 32 bits."""
    x, r = x.float(), 2 * co.shape[-1]
    if interleaved:
        u, v = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((u * co - v * si, v * co + u * si), -1).flatten(-2)
    else:
        u, v = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((u * co - v * si, v * co + u * si), -1)
    return torch.cat((turned, x[..., r:]), -1).to(torch.bfloat16)


def _rotary(st):
    c = st["c"]
    place = _where(st)[2] if st["places"] is None else st["places"]
    angle = place.double()[:, None] * st["inv_freq"]
    co, si = ((f * st["factor"]).float()[:, None] for f in (angle.cos(), angle.sin()))
    out = [_turned(x.detach(), co, si, c["interleaved"]) for x in (st["q"], st["k"])]
    if c["grad"]:  # turned back
        out += [_turned(x, co, -si, c["interleaved"]) for x in (st["gq"], st["gk"])]
    return tuple(out)


def _as_float(pages, scale):
    if scale is None:
        return pages.float()
    return pages.float() * scale[..., None, None]


def _read(st):
    c = st["c"]
    s, _, place = _where(st)
    page, slot = st["table"][s, place // c["page"]].long(), place % c["page"]

    def rows(pages, scale):
        if scale is None:
            return pages[page, :, slot]
        x = pages.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
        return (x * scale[page][..., None]).to(torch.bfloat16)
    return rows(st["k_pages"], st["k_scale"]), rows(st["v_pages"], st["v_scale"])


def _chunk(st):
    c = st["c"]
    S, N, L, hkv, g = c["seqs"], st["most"], st["longest"], c["hkv"], c["hq"] // c["hkv"]
    kv, cu = st["kv_len"].long(), st["cu"].long()
    n = cu.diff()
    i = torch.arange(N, device=DEV)
    q = st["q"][(cu[:-1, None] + i).clamp(max=st["tokens"] - 1)].float()
    q = q.view(S, N, hkv, g, D).transpose(1, 2).reshape(S, hkv, N * g, D)
    page = st["table"][:, :(L + c["page"] - 1) // c["page"]].clamp(min=0).long()

    def rows(pages, scale):
        x = _as_float(pages.view(torch.uint8)[page].view(pages.dtype) if scale is not None else pages[page], None if scale is None else scale[page])
        return x.transpose(1, 2).reshape(S, hkv, -1, D)[:, :, :L]
    k = rows(st["k_pages"], st["k_scale"])
    x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)
    del k
    place = (kv - n)[:, None] + i
    key = torch.arange(L, device=DEV)
    seen = key <= place[..., None]
    if c["window"]:
        seen &= key > place[..., None] - c["window"]
    seen = seen.repeat_interleave(g, 1)[:, None]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(3, keepdim=True)
    w = torch.exp(x - top)
    del x
    total = w.sum(3, keepdim=True)
    o = torch.matmul(w, rows(st["v_pages"], st["v_scale"])) / total
    s, i, _ = _where(st)
    o = o.view(S, hkv, N, g, D)[s, :, i].reshape(-1, c["hq"], D)
    lse = (top + total.log()).view(S, hkv, N, g)[s, :, i].reshape(-1, c["hq"])
    if c["gated"]:
        o = st["o_acc"].float() + st["gate"][..., None] * o
    return o.to(torch.bfloat16), lse


# ---- the definition in 64 bits, sequence by sequence ----------------------------------------------------------------------
def exact(case, seed):
    c = case
    st = prepare(c, seed)
    kv, new = _lengths(c)
    if c["op"] == "rotary":
        if st["places"] is None:
            place = torch.cat([torch.arange(x, dtype=torch.float64, device=DEV) for x in new])
        else:
            place = st["places"].double()

        def turned(x, sign):
            x = x.detach()
            y = x.double()
            for i in range(c["rot"] // 2):
                a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot"] // 2)
                angle = (place * st["inv_freq"][i] * sign)[:, None]
                u, v = x[..., a].double(), x[..., b].double()
                y[..., a] = (u * torch.cos(angle) - v * torch.sin(angle)) * st["factor"]
                y[..., b] = (v * torch.cos(angle) + u * torch.sin(angle)) * st["factor"]
            return y
        out = [turned(st["q"], 1), turned(st["k"], 1)]
        return tuple(out + ([turned(st["gq"], -1), turned(st["gk"], -1)] if c["grad"] else []))
    P, T, hkv = c["page"], sum(new), c["hkv"]

    def stored(pages, scale, s, j):
        """The values of head j of sequence s."""
        ids = st["table"][s, :(kv[s] + P - 1) // P].long()
        if scale is None:
            x = pages[ids, j].double()
        else:
            x = pages.view(torch.uint8)[ids, j].view(torch.float8_e4m3fn).double() * scale[ids, j].double()[:, None, None]
        return x.reshape(-1, D)[:kv[s]]
    if c["op"] == "read":
        out = [torch.empty(T, hkv, D, dtype=torch.float64, device=DEV) for _ in range(2)]
        t = 0
        for s in range(len(kv)):
            for j in range(hkv):
                out[0][t:t + kv[s], j] = stored(st["k_pages"], st["k_scale"], s, j)
                out[1][t:t + kv[s], j] = stored(st["v_pages"], st["v_scale"], s, j)
            t += kv[s]
        return tuple(out)
    g = c["hq"] // hkv
    o = torch.empty(T, c["hq"], D, dtype=torch.float64, device=DEV)
    lse = torch.empty(T, c["hq"], dtype=torch.float64, device=DEV)
    t = 0
    for s in range(len(kv)):
        n = new[s]
        last = torch.arange(kv[s] - n, kv[s], device=DEV).repeat_interleave(g)[:, None]
        for j in range(hkv):
            k, v = stored(st["k_pages"], st["k_scale"], s, j), stored(st["v_pages"], st["v_scale"], s, j)
            x = st["q"][t:t + n, j * g:(j + 1) * g].reshape(n * g, D).double() @ k.T * D ** -0.5
            u = torch.arange(kv[s], device=DEV)[None]
            x.masked_fill_((u > last) | (u <= last - (c["window"] or kv[s])), -math.inf)
            z = torch.logsumexp(x, 1)
            o[t:t + n, j * g:(j + 1) * g] = (x.sub_(z[:, None]).exp_() @ v).view(n, g, D)
            lse[t:t + n, j * g:(j + 1) * g] = z.view(n, g)
        t += n
    if c["gated"]:
        o = st["o_acc"].double() + st["gate"].double()[..., None] * o
    return o, lse
