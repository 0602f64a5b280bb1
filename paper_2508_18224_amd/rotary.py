"""Rotary positions for queries and keys of the training path (nsa_sel_rotary of include/nsa_sel.h, which states the rules).  Arguments are checked and handed to the
library in csrc/bind_cache.cpp, which has the gradient too; no arithmetic on tensors happens here."""
from __future__ import annotations

import math
from typing import Optional

import torch

from .binding import NsaSelError, call_native, native


def rotary(q: torch.Tensor, k: Optional[torch.Tensor], inv_freq: torch.Tensor, cu: Optional[torch.Tensor] = None, *,
           positions: Optional[torch.Tensor] = None, interleaved: bool = False, factor: float = 1.0, q_out: Optional[torch.Tensor] = None,
           k_out: Optional[torch.Tensor] = None):
    """(q, k) turned by their tokens' places; differentiable in q and k (backward; tensors with a forward gradient and tracing are refused).  q, k: bfloat16 [tokens, heads, 128] device tensors, any numbers of heads, that may be slices
    whose tokens lie apart (k may be None).  The bits are those that PagedCache.append writes.

    inv_freq: float64 [rot / 2], radians per place, rot a multiple of 16 up to 128 leading channels, and factor, which multiplies those channels: rotary_frequencies gives both.
    Pairs are channels (i, i + rot / 2), or (2 i, 2 i + 1) if interleaved.  The place of a token is its place in its sequence by cu (int32 [sequences + 1]; None: one
    sequence), or what positions (int32 [tokens]) says, beside which cu is not looked at.  Tokens of no sequence are copied as they are.

    q_out / k_out take the results where no gradient is wanted (they may be q / k themselves)."""
    if not isinstance(q, torch.Tensor):
        raise NsaSelError("q must be a torch.Tensor")
    node = q_out is None and k_out is None and torch.is_grad_enabled() and (q.requires_grad or (isinstance(k, torch.Tensor) and k.requires_grad))
    return call_native(native().rotary, q.device, q, k, inv_freq, cu, positions, interleaved, factor, False, q_out, k_out, node)


def rotary_frequencies(rot: int = 128, base: float = 10000.0, *, scaling: Optional[str] = None, stretch: float = 1.0, trained: int = 8192,
                       fast: float = 32.0, slow: float = 1.0, device="cuda:0"):
    """(inv_freq, factor) for rotary and PagedCache.append: float64 [rot / 2] radians per place, base ** (-2 i / rot), changed for a context `stretch` times as long as the
    `trained` one:
      scaling None       not
      "linear"           all divided by stretch
      "base"             base raised so that the slowest pair is stretched by `stretch` and the fastest not at all
      "parts"            pairs that turn more than `fast` times within `trained` places as they are, those that turn less than `slow` times divided by stretch, those in
                         between a mean of both by the number of turns; factor 0.1 log(stretch) + 1 for both queries and keys (Peng et al., arXiv 2309.00071)
    """
    if rot < 16 or rot > 128 or rot % 16 or not base > 1 or not stretch >= 1 or not fast > slow >= 0 or trained < 1:
        raise NsaSelError("rot must be a multiple of 16 up to 128, base above 1, stretch at least 1, fast above slow, trained positive")
    if scaling not in (None, "linear", "base", "parts"):
        raise NsaSelError(f"scaling must be None, 'linear', 'base' or 'parts', got {scaling!r}")
    factor = 1.0
    if scaling == "base":
        base = base * stretch ** (rot / (rot - 2))
    out = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        out = [f / stretch for f in out]
    elif scaling == "parts":
        keep = [min(1.0, max(0.0, (trained * f / (2 * math.pi) - slow) / (fast - slow))) for f in out]
        out = [f * (k + (1 - k) / stretch) for f, k in zip(out, keep)]
        factor = 0.1 * math.log(stretch) + 1.0
    return torch.tensor(out, dtype=torch.float64, device=device), factor
