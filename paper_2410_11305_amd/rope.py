"""Rotary frequencies of a model, worked out once on the host: what rope_kv4_append takes as inv_freq and mscale.

Pair i of a head's first `rot` features turns by inv_freq[i] radians per position, theta^(-2i/rot) for a model that
runs at the length it was trained on.  For contexts `factor` times longer than `original` positions:
  linear  every frequency divided by factor (positions squeezed into the trained range)
  ntk     theta raised to theta * factor^(rot / (rot - 2)): the slowest pair turns factor times slower, the fastest as before
  yarn    pairs with fewer than `slow` turns over the trained length divided by factor, those with more than `fast` left
          alone, a linear blend in between (over the index of the pair, from whole index to whole index); queries and keys scaled by 0.1 ln(factor) + 1
"""
from __future__ import annotations

import math

import torch


def frequencies(rot: int, theta: float = 10000.0, scaling: str = None, factor: float = 1.0, original: int = 4096,
                fast: float = 32.0, slow: float = 1.0, device="cuda"):
    """(inv_freq float64 [rot/2] on `device`, mscale)."""
    if rot < 2 or rot % 2 or not theta > 1.0:
        raise ValueError(f"rot must be even and positive and theta above 1, got {rot} and {theta}")
    if scaling not in (None, "linear", "ntk", "yarn"):
        raise ValueError(f"scaling must be None, 'linear', 'ntk' or 'yarn', got {scaling!r}")
    if scaling is not None and not (factor >= 1.0 and math.isfinite(factor)):
        raise ValueError(f"factor must be 1 or more, got {factor}")
    if scaling == "ntk":
        if rot < 4:
            raise ValueError("ntk scaling needs two pairs or more")
        theta = theta * factor ** (rot / (rot - 2))
    inv = [theta ** (-2.0 * i / rot) for i in range(rot // 2)]
    mscale = 1.0
    if scaling == "linear":
        inv = [f / factor for f in inv]
    elif scaling == "yarn":
        if original < 1 or not fast > slow > 0.0:
            raise ValueError("yarn scaling needs original >= 1 and fast > slow > 0")
        # index of the pair that makes n turns over the trained length
        index = lambda n: rot * math.log(original / (n * 2.0 * math.pi)) / (2.0 * math.log(theta))
        # (past the last pair, rot / 2 - 1, where all of them make `slow` turns: the line to there is not squeezed)
        low, high = max(math.floor(index(fast)), 0), min(math.ceil(index(slow)), rot - 1)
        for i in range(rot // 2):
            squeezed = min(max((i - low) / max(high - low, 1e-3), 0.0), 1.0)
            inv[i] = inv[i] * (1.0 - squeezed) + inv[i] / factor * squeezed
        mscale = 0.1 * math.log(factor) + 1.0
    return torch.tensor(inv, dtype=torch.float64, device=device), mscale
