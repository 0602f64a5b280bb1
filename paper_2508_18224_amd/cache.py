"""A paged cache of keys and values and the calls over it (the nsa_sel_cache_* part of include/nsa_sel.h, which states the rules).  Arguments are checked and
handed to the library in csrc/bind_cache.cpp; no arithmetic happens here."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import CacheShape, NsaSelError, _check, _device, call_native, lib, native

_BF16 = torch.bfloat16
_D = 128


class PagedCache:
    """Pages of keys and values, [n_pages, hkv, page, 128] each, in bfloat16 or torch.float8_e4m3fn; in the latter with one power-of-two
    scale for every (page, KV head).  Which pages a sequence has is the caller's: `table` (int32 [sequences, max_pages], page ids, -1 for
    none) and `kv_len` (int32 [sequences], lengths INCLUDING the new tokens) go with every call.  The new tokens of all sequences are
    packed, their starts in `cu` (int32 [sequences + 1]); cu = None: one new token for each sequence.

    A step of a layer is append, selection, attention:

        q, _ = cache.append(k, v, table, kv_len, q=q, inv_freq=inv_freq)
        idx = select_blocks(scores, None, topk, kv_len=kv_len)
        o, lse = cache.attention(q, table, kv_len, idx=idx)

    Forward only: in grad mode tensors that require grad are refused.  Calls keep nothing between them and may run on any stream and be captured; calls that write the same pages at once
    race, as writes to any tensor do.

    k_pages, v_pages, k_scale, v_scale (None in bfloat16), n_pages, hkv, page and device are there to be read.  The tensors are looked at in every call:
    their owner may give them other storage in between, of the same shape.  A larger cache is another PagedCache."""

    def __init__(self, n_pages: int, hkv: int, *, page: int = 64, dtype: torch.dtype = _BF16, device="cuda:0"):
        device = _device(device)
        if dtype not in (_BF16, torch.float8_e4m3fn):
            raise NsaSelError(f"pages must be bfloat16 or float8_e4m3fn, got {dtype}")

        def zeros():
            bits = torch.int16 if dtype is _BF16 else torch.uint8
            return torch.zeros((n_pages, hkv, page, _D), dtype=bits, device=device).view(dtype)
        scales = (None, None) if dtype is _BF16 else (torch.ones((n_pages, hkv), device=device) for _ in range(2))
        self._set(zeros(), zeros(), *scales)

    @classmethod
    def from_tensors(cls, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                     v_scale: Optional[torch.Tensor] = None) -> "PagedCache":
        """A cache in the caller's own tensors."""
        self = cls.__new__(cls)
        self._set(k_pages, v_pages, k_scale, v_scale)
        return self

    def _set(self, k_pages, v_pages, k_scale, v_scale):
        self._calls = native()
        self._info = self._calls.describe(k_pages, v_pages, k_scale, v_scale)
        self._tensors = (k_pages, v_pages, k_scale, v_scale)
        self._sizes = tuple(k_pages.shape[:3])
        self._device = k_pages.device

    k_pages = property(lambda self: self._tensors[0])
    v_pages = property(lambda self: self._tensors[1])
    k_scale = property(lambda self: self._tensors[2])
    v_scale = property(lambda self: self._tensors[3])
    n_pages = property(lambda self: self._sizes[0])
    hkv = property(lambda self: self._sizes[1])
    page = property(lambda self: self._sizes[2])
    device = property(lambda self: self._device)

    def append(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, cu: Optional[torch.Tensor] = None, *,
               q: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, interleaved: bool = False,
               rotated_k: bool = False, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """Writes k and v (bfloat16 [tokens, hkv, 128]) to the pages, k rotated by its tokens' places, and returns (rotated q or None,
        rotated k as bfloat16 or None).  q, k, v may be slices whose tokens lie apart.

        inv_freq: float64 [rot / 2], radians per place, rot a multiple of 16 up to 128 leading channels; None rotates nothing.  Pairs are
        channels (i, i + rot / 2), or (2 i, 2 i + 1) if interleaved.  rotated_k also returns the rotated keys, for the prompt's own
        attention.  q_out / k_out take the results (they may be q / k themselves if those are contiguous); rows of tokens that belong to no
        sequence, and of tokens of negative place (idle slots, with kv_len 0), are left as they are there, and uninitialised otherwise: attention looks at
        neither."""
        return call_native(self._calls.append, self._device, self._info, k, v, table, kv_len, cu, q, inv_freq, interleaved, rotated_k, q_out, k_out)

    def workspace_bytes(self, tokens: int, hq: int, nseq: int, max_pages: int, *, topk: int = 0, block: int = 64, window: int = 0) -> int:
        """Bytes that attention() of such a call needs as `ws`."""
        for name, x in dict(tokens=tokens, hq=hq, nseq=nseq, max_pages=max_pages, topk=topk, block=block, window=window).items():
            if not -2 ** 31 <= x < 2 ** 31:
                raise NsaSelError(f"{name} is out of range")
        shape = CacheShape(tokens, nseq, hq, self.hkv, _D, int(self.k_pages.dtype is not _BF16), self.page, self.n_pages, max_pages, block, topk, window, 0.0)
        need = C.c_size_t()
        _check(lib().nsa_sel_cache_workspace_bytes(C.byref(shape), C.byref(need)), "nsa_sel_cache_workspace_bytes")
        return need.value

    def attention(self, q: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, cu: Optional[torch.Tensor] = None, *,
                  idx: Optional[torch.Tensor] = None, block: int = 64, window: int = 0, scale: float = 0.0,
                  gate: Optional[torch.Tensor] = None, o_acc: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
        """(O, LSE) of the new tokens' queries (bfloat16 [tokens, hq, 128], rotated) over the cache, their own keys included: over the
        blocks of `idx` (int32 [tokens, hkv, topk]; select_blocks with kv_len gives it), over the last `window` places, over both, or over
        every key.  With gate (float32 [tokens, hq]) O is o_acc + gate * O, the sum over a layer's branches.

        out / lse take the results (out may be o_acc); rows of tokens that belong to no sequence are left as they are there, and
        uninitialised otherwise.  ws, of workspace_bytes(), is for callers that may not allocate."""
        return call_native(self._calls.attention, self._device, self._info, q, table, kv_len, cu, idx, block, window, scale, gate, o_acc, out, lse, ws)
