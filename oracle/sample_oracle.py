"""CPU oracle for sampling from given random numbers and the acceptance walk over sampled tokens.

TEST INFRASTRUCTURE ONLY.  Plain Python floats (binary64), one token after another; shares no code with the HIP path.

Definition: the tokens of a row by falling logit, the lowest id first among equals; w = exp((logit - max) /
temperature); top_k keeps the first top_k, min_p those with w >= min_p, top_p the shortest beginning of the rest that
holds top_p of its mass; the token is the first whose running mass exceeds u times the mass kept.  temperature <= 0: the
first of that order.  -inf and NaN are never chosen (token -1 if there is nothing else); +inf outweighs every number.
"""
from __future__ import annotations

import math

import numpy as np


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) -> int:
    x = [float(v) for v in np.asarray(row).tolist()]
    order = sorted((i for i in range(len(x)) if x[i] > -math.inf), key=lambda i: (-x[i], i))      # (NaN compares false)
    if not order:
        return -1
    if not temperature > 0:
        return order[0]
    top = x[order[0]]
    weight = lambda v: 1.0 if v == top else 0.0 if top == math.inf else math.exp(max((v - top) / temperature, -745.0)) if (v - top) / temperature > -745.0 else 0.0
    w = [weight(x[i]) for i in order]
    n = len(w)
    if top_k > 0:
        n = min(n, top_k)
    if min_p > 0:
        n = min(n, sum(1 for a in w if a >= min(min_p, 1.0)))
    if top_p < 1:
        limit, mass, kept = top_p * math.fsum(w[:n]), 0.0, 0
        while kept < n and (kept == 0 or mass < limit):
            mass += w[kept]
            kept += 1
        n = kept
    target = min(max(u, 0.0), 0.99999994) * math.fsum(w[:n])
    mass, last = 0.0, order[0]
    for a, i in zip(w[:n], order):
        mass += a
        if a > 0:
            last = i
        if mass > target:
            return i
    return last


def accept(tokens, draft):
    """tokens [B, gamma+1] chosen by the verify pass, draft [B, gamma] -> (n_accept [B], out_tokens [B, gamma+1])."""
    B, rows = tokens.shape
    n, out = np.zeros(B, dtype=np.int32), np.full((B, rows), -1, dtype=np.int32)
    for b in range(B):
        while n[b] < rows - 1 and tokens[b, n[b]] == draft[b, n[b]]:
            n[b] += 1
        out[b, :n[b] + 1] = tokens[b, :n[b] + 1]
    return n, out
