"""CPU oracle for the choice of pages of the 4-bit cache, and for attention over chosen pages.

TEST INFRASTRUCTURE ONLY.  Plain NumPy from the definitions; shares no code with the HIP path.

Definitions (all of them this library's):
  bounds     per page, head and feature the largest and smallest key value code * step + low, rounded to binary32, of the page's
             tokens; in whole numbers of a grid, rounded outward, the grid the smallest power of two that keeps all
             features within +-127 (1 for zeros).  A step or low that is no finite number: codes 0, grid NaN
  score      grid * max over the heads of a key/value head of sum_d max(c upper, c lower), c the row's queries in whole numbers, to nearest even,
             of their own such grid (zeros if one of them is no finite number)
  choice     the first and last pages in sight, then the best; the lower page among equals; NaN grids before all others, absent pages last
"""
from __future__ import annotations

import numpy as np


def grid_of(top: float) -> float:
    if top == 0:
        return 1.0
    e = -160
    while top > 127.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def bounds(codes, step, low):
    """Keys of some tokens, codes [tokens, D] with step, low fp16 [tokens] -> (upper int8 [D], lower int8 [D], grid)."""
    D = codes.shape[1]
    if not (np.isfinite(step).all() and np.isfinite(low).all()):
        return np.zeros(D, np.int8), np.zeros(D, np.int8), np.float32(np.nan)
    x = (codes.astype(np.float64) * step.astype(np.float64)[:, None] + low.astype(np.float64)[:, None]).astype(np.float32).astype(np.float64)
    upper, lower = x.max(0), x.min(0)
    grid = grid_of(max(np.abs(upper).max(), np.abs(lower).max()))
    return np.ceil(upper / grid).astype(np.int8), np.floor(lower / grid).astype(np.int8), np.float32(grid)


def bounds_bytes(upper, lower, grid) -> np.ndarray:
    """Codes int8 [pages, Hkv, D] and grids fp32 [pages, Hkv] -> the bounds' bytes."""
    n, H, D = upper.shape
    rows = np.concatenate((upper, lower), -1).astype(np.int8).reshape(n, H * 2 * D).view(np.uint8)
    grids = np.ascontiguousarray(grid.astype(np.float32)).view(np.uint8).reshape(n, 4 * H)
    return np.concatenate((rows, grids, np.zeros((n, -4 * H % 16), np.uint8)), -1)


def query_codes(q) -> np.ndarray:
    """The heads of one row and key/value head, fp16 [G, D] -> whole numbers [G, D]."""
    x = q.astype(np.float64)
    if not np.isfinite(x).all():
        return np.zeros(x.shape, np.int64)
    return np.rint(x / grid_of(np.abs(x).max())).astype(np.int64)


def scores(q, upper, lower, grid, there) -> np.ndarray:
    """q fp16 [G, D]; upper, lower [n, D], grid [n], there bool [n] -> binary64 [n], infinite where a page is taken or left in any case."""
    c = query_codes(q)
    u, l = upper.astype(np.int64), lower.astype(np.int64)
    dots = np.maximum(c, 0) @ u.T + np.minimum(c, 0) @ l.T
    with np.errstate(invalid="ignore"):
        s = dots.max(0) * grid.astype(np.float64)
    return np.where(there, np.where(np.isnan(grid), np.inf, s), -np.inf)


def choose(score, first, last, count):
    """score [n] of the pages in sight -> int32 [count], ascending, -1 behind the last."""
    n = len(score)
    forced = [i for i in range(n) if i < first or i >= n - last]
    rest = sorted((i for i in range(n) if not (i < first or i >= n - last)), key=lambda i: (-score[i], i))
    best = sorted((forced + rest)[:count]) if n > count else list(range(n))
    return np.array(best + [-1] * (count - len(best)), dtype=np.int32)


def in_sight(position: int, P: int, max_pages: int) -> int:
    return 0 if position < 0 else min(position // P + 1, max_pages)


def listed(pages, n, max_pages) -> list:
    """The pages of a list that count, of a row that sees n pages."""
    out, before = [], -1
    for e in pages[:max(min(len(pages), n), 1)]:
        if 0 <= e < max_pages and e > before:
            out.append(int(e))
        before = e
    return out
