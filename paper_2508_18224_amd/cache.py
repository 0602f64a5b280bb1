"""A paged cache of keys and values and the calls over it (the nsa_sel_cache_* part of include/nsa_sel.h, which states the rules).  Like
binding.py this marshals and checks arguments; no arithmetic happens here."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from .binding import CacheShape, NsaSelError, _check, _device, _launch, _ptr, expect_tensor, expect_workspace, lib

# A decoding loop calls these a few times a layer with a few tokens: what a call costs on the host is what it costs.  So a tensor is looked at
# once, and what follows from the sizes of a call alone is kept for the next call of the same sizes.

_BF16, _F32, _I32, _F64 = torch.bfloat16, torch.float32, torch.int32, torch.float64
_D = 128


def _rows(name: str, t, shape, device) -> int:
    """Values between the tokens of a bf16 [tokens, heads, 128] tensor.  They may lie apart (a slice of one projection), its heads may not."""
    if not isinstance(t, torch.Tensor):
        raise NsaSelError(f"{name} must be a torch.Tensor")
    if t.dtype is not _BF16 or t.shape != shape:
        raise NsaSelError(f"{name} must be bfloat16 {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.device != device:
        raise NsaSelError(f"{name} must live on {device}, got {t.device}")
    tokens, heads, _ = shape
    if t.data_ptr() & 15:
        raise NsaSelError(f"{name} must be 16-byte aligned")
    if t.is_contiguous():
        return heads * _D
    each, head, one = t.stride()
    if one != 1 or (heads > 1 and head != _D):
        raise NsaSelError(f"the heads of a token of {name} must be contiguous")
    if tokens > 1 and (each < heads * _D or each & 7):
        raise NsaSelError(f"the tokens of {name} must be a multiple of 8 values apart, and not overlap")
    return each if tokens > 1 else heads * _D


class PagedCache:
    """Pages of keys and values, [n_pages, hkv, page, 128] each, in bfloat16 or torch.float8_e4m3fn; in the latter with one power-of-two
    scale for every (page, KV head).  Which pages a sequence has is the caller's: `table` (int32 [sequences, max_pages], page ids, -1 for
    none) and `kv_len` (int32 [sequences], lengths INCLUDING the new tokens) go with every call.  The new tokens of all sequences are
    packed, their starts in `cu` (int32 [sequences + 1]); cu = None: one new token for each sequence.

    A step of a layer is append, selection, attention:

        q, _ = cache.append(k, v, table, kv_len, q=q, inv_freq=inv_freq)
        idx = select_blocks(scores, None, topk, kv_len=kv_len)
        o, lse = cache.attention(q, table, kv_len, idx=idx)

    Forward only.  Calls keep nothing between them and may run on any stream and be captured; calls that write the same pages at once
    race, as writes to any tensor do."""

    def __init__(self, n_pages: int, hkv: int, *, page: int = 64, dtype: torch.dtype = _BF16, device="cuda:0"):
        device = _device(device)
        if dtype not in (_BF16, torch.float8_e4m3fn):
            raise NsaSelError(f"pages must be bfloat16 or float8_e4m3fn, got {dtype}")

        def zeros():
            bits = torch.int16 if dtype is _BF16 else torch.uint8
            return torch.zeros((n_pages, hkv, page, _D), dtype=bits, device=device).view(dtype)
        scales = (None, None) if dtype is _BF16 else (torch.ones((n_pages, hkv), dtype=_F32, device=device) for _ in range(2))
        self._set(zeros(), zeros(), *scales)

    @classmethod
    def from_tensors(cls, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                     v_scale: Optional[torch.Tensor] = None) -> "PagedCache":
        """A cache in the caller's own tensors."""
        self = cls.__new__(cls)
        self._set(k_pages, v_pages, k_scale, v_scale)
        return self

    def _set(self, k_pages, v_pages, k_scale, v_scale):
        if not isinstance(k_pages, torch.Tensor) or k_pages.dtype not in (_BF16, torch.float8_e4m3fn) or k_pages.dim() != 4:
            raise NsaSelError("pages must be bfloat16 or float8_e4m3fn [n_pages, hkv, page, 128]")
        n_pages, hkv, page, d = k_pages.shape
        if d != _D or page not in (16, 32, 64, 128, 256) or hkv < 1:
            raise NsaSelError(f"pages must be [n_pages, hkv, page, {_D}] with 16, 32, 64, 128 or 256 tokens a page, got {tuple(k_pages.shape)}")
        expect_tensor("k_pages", k_pages, k_pages.dtype, k_pages.shape, k_pages.device)
        expect_tensor("v_pages", v_pages, k_pages.dtype, k_pages.shape, k_pages.device)
        e4m3 = k_pages.dtype is not _BF16
        if e4m3:
            expect_tensor("k_scale", k_scale, _F32, (n_pages, hkv), k_pages.device)
            expect_tensor("v_scale", v_scale, _F32, (n_pages, hkv), k_pages.device)
        elif k_scale is not None or v_scale is not None:
            raise NsaSelError("bfloat16 pages have no scales")
        self.k_pages, self.v_pages, self.k_scale, self.v_scale = k_pages, v_pages, k_scale, v_scale
        self.n_pages, self.hkv, self.page, self.device = n_pages, hkv, page, k_pages.device
        self._dtype = 1 if e4m3 else 0
        self._pointers = tuple(_ptr(t) for t in (k_pages, v_pages, k_scale, v_scale))
        self._shapes = {}  # sizes of a call -> (its shape, bytes of its workspace)

    def _batch(self, tokens: int, table, kv_len, cu) -> Tuple[int, int]:
        """(sequences, columns of table) after the checks that all calls share."""
        dev = self.device
        try:
            nseq, max_pages = table.shape
        except (AttributeError, ValueError):
            raise NsaSelError("table must be int32 [sequences, max_pages]") from None
        expect_tensor("table", table, _I32, (nseq, max_pages), dev)
        expect_tensor("kv_len", kv_len, _I32, (nseq,), dev)
        if cu is not None:
            expect_tensor("cu_seqlens", cu, _I32, (nseq + 1,), dev)
        elif nseq != tokens:
            raise NsaSelError(f"without cu_seqlens every sequence has one new token: {nseq} sequences for {tokens} tokens")
        return nseq, max_pages

    def _shape(self, tokens, nseq, hq, max_pages, block=64, topk=0, window=0, scale=0.0):
        """The shape of a call, to be passed on, and the bytes of the attention's workspace."""
        key = (tokens, nseq, hq, max_pages, block, topk, window, scale)
        known = self._shapes.get(key)
        if known is None:
            if not (0 <= window < 2 ** 31 and 0 < block < 2 ** 31):
                raise NsaSelError(f"window must be 0 or a number of tokens and block 64 or 128, got {window} and {block}")
            shape = CacheShape(tokens, nseq, hq, self.hkv, _D, self._dtype, self.page, self.n_pages, max_pages, block, topk, window, scale)
            need = C.c_size_t()
            _check(lib().nsa_sel_cache_workspace_bytes(C.byref(shape), C.byref(need)), "nsa_sel_cache_workspace_bytes")
            if len(self._shapes) >= 4096:
                self._shapes.clear()
            known = self._shapes[key] = (C.byref(shape), need.value)
        return known

    def append(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, cu: Optional[torch.Tensor] = None, *,
               q: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, interleaved: bool = False,
               rotated_k: bool = False, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """Writes k and v (bfloat16 [tokens, hkv, 128]) to the pages, k rotated by its tokens' places, and returns (rotated q or None,
        rotated k as bfloat16 or None).  q, k, v may be slices whose tokens lie apart.

        inv_freq: float64 [rot / 2], radians per place, rot a multiple of 16 up to 128 leading channels; None rotates nothing.  Pairs are
        channels (i, i + rot / 2), or (2 i, 2 i + 1) if interleaved.  rotated_k also returns the rotated keys, for the prompt's own
        attention.  q_out / k_out take the results (they may be q / k themselves if those are contiguous); rows of tokens that belong to no
        sequence are left as they are there, and uninitialised otherwise."""
        dev, hkv = self.device, self.hkv
        try:
            T = k.shape[0]
        except (AttributeError, IndexError):
            raise NsaSelError("k must be bfloat16 [tokens, hkv, 128]") from None
        kv_rows = (T, hkv, _D)
        k_stride, v_stride = _rows("k", k, kv_rows, dev), _rows("v", v, kv_rows, dev)
        nseq, max_pages = self._batch(T, table, kv_len, cu)
        hq, rot, q_stride, q_ptr = hkv, 0, 0, None
        if q is not None:
            try:
                _, hq, _ = q.shape
            except (AttributeError, ValueError):
                raise NsaSelError("q must be bfloat16 [tokens, hq, 128]") from None
            rows = (T, hq, _D)
            q_stride, q_ptr = _rows("q", q, rows, dev), q.data_ptr()
            if q_out is None:
                q_out = torch.empty_like(q) if q_stride == hq * _D else torch.empty(rows, dtype=_BF16, device=dev)
            else:
                expect_tensor("q_out", q_out, _BF16, rows, dev)
        elif q_out is not None:
            raise NsaSelError("q_out without q")
        if k_out is not None:
            expect_tensor("k_out", k_out, _BF16, kv_rows, dev)
        elif rotated_k:
            k_out = torch.empty(kv_rows, dtype=_BF16, device=dev)
        if inv_freq is not None:
            try:
                pairs, = inv_freq.shape
            except (AttributeError, ValueError):
                raise NsaSelError("inv_freq must be float64 [rot / 2]") from None
            expect_tensor("inv_freq", inv_freq, _F64, (pairs,), dev)
            rot = 2 * pairs
        _launch(lib().nsa_sel_cache_append, "nsa_sel_cache_append", dev, self._shape(T, nseq, hq, max_pages)[0], q_ptr, q_stride, k.data_ptr(), k_stride,
                v.data_ptr(), v_stride, _ptr(cu), kv_len.data_ptr(), table.data_ptr(), _ptr(inv_freq), rot, int(interleaved),
                *self._pointers, _ptr(q_out), _ptr(k_out))
        return q_out, k_out

    def workspace_bytes(self, tokens: int, hq: int, nseq: int, max_pages: int, *, topk: int = 0, block: int = 64, window: int = 0) -> int:
        """Bytes that attention() of such a call needs as `ws`."""
        return self._shape(tokens, nseq, hq, max_pages, block, topk, window)[1]

    def attention(self, q: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, cu: Optional[torch.Tensor] = None, *,
                  idx: Optional[torch.Tensor] = None, block: int = 64, window: int = 0, scale: float = 0.0,
                  gate: Optional[torch.Tensor] = None, o_acc: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
        """(O, LSE) of the new tokens' queries (bfloat16 [tokens, hq, 128], rotated) over the cache, their own keys included: over the
        blocks of `idx` (int32 [tokens, hkv, topk]; select_blocks with kv_len gives it), over the last `window` places, over both, or over
        every key.  With gate (float32 [tokens, hq]) O is o_acc + gate * O, the sum over a layer's branches.

        out / lse take the results (out may be o_acc); rows of tokens that belong to no sequence are left as they are there, and
        uninitialised otherwise.  ws, of workspace_bytes(), is for callers that may not allocate."""
        dev = self.device
        try:
            T, hq, _ = q.shape
        except (AttributeError, ValueError):
            raise NsaSelError("q must be bfloat16 [tokens, hq, 128]") from None
        rows = (T, hq, _D)
        expect_tensor("q", q, _BF16, rows, dev)
        nseq, max_pages = self._batch(T, table, kv_len, cu)
        topk = 0
        if idx is not None:
            try:
                _, _, topk = idx.shape
            except (AttributeError, ValueError):
                topk = 0
            if topk < 1:
                raise NsaSelError("idx must be int32 [tokens, hkv, topk], topk at least 1")
            expect_tensor("idx", idx, _I32, (T, self.hkv, topk), dev)
        if gate is not None:
            expect_tensor("gate", gate, _F32, (T, hq), dev)
            if o_acc is not None:
                expect_tensor("o_acc", o_acc, _BF16, rows, dev)
        elif o_acc is not None:
            raise NsaSelError("o_acc without gate")
        if out is None:
            out = torch.empty_like(q)
        else:
            expect_tensor("out", out, _BF16, rows, dev)
        if lse is None:
            lse = torch.empty((T, hq), dtype=_F32, device=dev)
        else:
            expect_tensor("lse", lse, _F32, (T, hq), dev)
        shape, need = self._shape(T, nseq, hq, max_pages, block, topk, window, scale)
        if ws is not None:
            expect_workspace("ws", ws, need, dev)
        elif need:
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
        _launch(lib().nsa_sel_cache_attention, "nsa_sel_cache_attention", dev, shape, q.data_ptr(), _ptr(idx), _ptr(cu),
                kv_len.data_ptr(), table.data_ptr(), *self._pointers, _ptr(gate), _ptr(o_acc), out.data_ptr(), lse.data_ptr(), _ptr(ws),
                0 if ws is None else need)
        return out, lse
