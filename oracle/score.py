"""Attention with capped scores, distance biases and masks, in float64."""
from __future__ import annotations

from typing import Optional

import numpy as np


def seen(p: np.ndarray, n: int, causal: bool = False, window: int = 0, prefix: int = 0,
         q_docs: Optional[np.ndarray] = None, k_docs: Optional[np.ndarray] = None) -> np.ndarray:
    """[queries, n]: whether a query at position p[i] sees key j."""
    out = np.zeros((len(p), n), dtype=bool)
    for i, at in enumerate(p):
        for lo, hi in [(0 if not window else at - window + 1, at if causal else at + window - 1 if window else n - 1), (0, prefix - 1)]:
            lo, hi = max(lo, 0), min(hi, n - 1)
            if lo <= hi:
                out[i, lo:hi + 1] = True
    if q_docs is not None:
        out &= (q_docs[:, None] == k_docs[None, :n]) & (q_docs[:, None] >= 0)
    return out


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, see: np.ndarray, p: np.ndarray, scale: float, cap: float = 0.0,
           slope: float = 0.0):
    """One head: q [Tq, d] at positions p over k, v [n, d].  Returns the output, sum p |v|
    per output, and what the scores of each query are made of: the largest sum |q k|
    scale and the largest |score|, distance's share included, among the keys it sees."""
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    some = see.any(1)
    out, A = np.zeros_like(q), np.zeros_like(q)
    size, mag = np.zeros(len(q)), np.zeros(len(q))
    for i in np.nonzero(some)[0]:
        j = np.nonzero(see[i])[0]
        s = (k[j] @ q[i]) * scale
        size[i] = (np.abs(k[j]) @ np.abs(q[i])).max() * scale
        if cap:
            s = cap * np.tanh(s / cap)
        far = slope * np.abs(p[i] - j)
        mag[i] = (np.abs(s) + np.abs(far)).max()
        s = s - far
        w = np.exp(s - s.max())
        w /= w.sum()
        with np.errstate(invalid="ignore"):
            out[i] = (w[:, None] * v[j]).sum(0)
            A[i] = (w[:, None] * np.abs(v[j])).sum(0)
    return out, A, size, mag
