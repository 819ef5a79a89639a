"""CPU oracle for the 4-bit key/value cache: rotary positions, the quantised append, the cache's bytes, and attention
over it.

TEST INFRASTRUCTURE ONLY.  Plain NumPy in binary64 from the definitions; shares no code with the HIP path.

Definitions (the paper fixes only that one cache serves both passes and that the verify pass overwrites the draft
pass's entries, Sec. 3.1; the 4-bit form is this library's):
  rotation   pair (a, b) at position p: mscale (a cos t - b sin t), mscale (b cos t + a sin t), t = p inv_freq[i],
             rounded once to fp16; pairs (i, i + rot/2) or (2i, 2i + 1)
  codes      per token and head: low = min x, step = fp16((max x - low) / 15), code = clamp(rne((x - low) / step), 0, 15)
             with the quotient in rational arithmetic (half way: to even); step 0: code 0.  A row with a NaN or an infinity:
             step and low NaN, codes 0
  attention  softmax(scale q k) v over the tokens in the cache at t <= p, inside the window or among the sinks; a row
             that sees nothing gives zeros

Cache bytes: see `cache_bytes`, which builds them code by code.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, interleaved: bool, mscale: float = 1.0) -> np.ndarray:
    """x fp16 [N, H, D], positions [N] -> fp16 [N, H, D]."""
    rot = 2 * len(inv_freq)
    y = x.astype(np.float64)
    out = x.copy()
    for i, f in enumerate(inv_freq):
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        t = positions.astype(np.float64) * f
        c, s = (np.cos(t) * mscale)[:, None], (np.sin(t) * mscale)[:, None]
        out[:, :, ia] = (y[:, :, ia] * c - y[:, :, ib] * s).astype(np.float16)
        out[:, :, ib] = (y[:, :, ib] * c + y[:, :, ia] * s).astype(np.float16)
    return out


def quantise(x: np.ndarray):
    """x fp16 [..., D] -> (codes uint8 [..., D], step fp16 [...], low fp16 [...])."""
    number = np.isfinite(x).all(-1)
    y = np.where(number[..., None], x.astype(np.float64), 0.0)
    low = y.min(-1) + 0.0                                     # a zero is +0
    step = ((y.max(-1) + 0.0 - low) / 15.0).astype(np.float16)
    s = step.astype(np.float64)[..., None]
    quotient = (y - low[..., None]) / np.where(s > 0, s, 1.0)
    codes = np.where(s > 0, np.clip(np.rint(quotient), 0, 15), 0).astype(np.uint8)
    return codes, np.where(number, step, np.float16(np.nan)), np.where(number, low.astype(np.float16), np.float16(np.nan))


def quantise_exactly(x) -> list:
    """The codes of one row in rational arithmetic."""
    v = [Fraction(float(e)) for e in x]
    low = min(v)
    step = Fraction(float(np.float16(float(max(v) - low) / 15.0)))
    return [min(max(round((e - low) / step), 0), 15) if step else 0 for e in v]


def nibble(e: int) -> int:
    """Position of code e of a run of 8 inside its word."""
    return {0: 0, 2: 1, 4: 2, 6: 3, 1: 4, 3: 5, 5: 6, 7: 7}[e]


def cache_bytes(k, ks, kl, v, vs, vl, page_size: int) -> np.ndarray:
    """Codes uint8 [n_pages, Hkv, P, D] and step, low fp16 [n_pages, Hkv, P] of keys and values -> the cache, uint8
    [n_pages, Hkv * P * (D + 8)]."""
    n, H, P, D = k.shape
    assert P == page_size
    words = np.zeros((2, n, H, P, D // 8), dtype=np.uint32)
    for which, codes in enumerate((k, v)):
        for e in range(8):
            words[which] |= codes[..., e::8].astype(np.uint32) << np.uint32(4 * nibble(e))
    value_tiles = words[1].reshape(n, H, P // 16, 16, D // 8).swapaxes(-1, -2)         # word, then token of the tile
    rows = np.stack((ks, kl, vs, vl), -1).astype(np.float16)
    out = np.concatenate([np.ascontiguousarray(a).reshape(n, H, -1).view(np.uint8) for a in (words[0], value_tiles, rows)], axis=-1)
    return out.reshape(n, -1)


def values(codes, step, low) -> np.ndarray:
    return codes.astype(np.float64) * step.astype(np.float64)[..., None] + low.astype(np.float64)[..., None]


def visible(position: int, tokens: int, window: int, sinks: int) -> np.ndarray:
    t = np.arange(tokens)
    seen = t <= position
    if window:
        seen &= (t > position - window) | (t < sinks)
    return seen


def attention(q, k, v, present, positions, scale, window=0, sinks=0) -> np.ndarray:
    """One sequence: q fp16 [T, Hq, D], k and v binary64 [tokens, Hkv, D], present bool [tokens] (in the cache), positions
    [T] -> binary64 [T, Hq, D]."""
    T, Hq, D = q.shape
    group = Hq // k.shape[1]
    out = np.zeros((T, Hq, D))
    for j in range(T):
        seen = visible(int(positions[j]), k.shape[0], window, sinks) & present
        if not seen.any():
            continue
        for h in range(Hq):
            s = (k[seen, h // group] @ q[j, h].astype(np.float64)) * scale
            w = np.exp(s - s.max())
            out[j, h] = (w @ v[seen, h // group]) / w.sum()
    return out
