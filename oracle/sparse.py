"""Attention over selected key blocks, in float64.

Blocks of 128 queries and of 64 keys.  A key block's score for a query block is
the product of their means; the best `keep` are listed in ascending order.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np

QB, KB = 128, 64


def _means(x: np.ndarray, size: int) -> np.ndarray:
    """[T, d] -> means of the blocks of `size` rows."""
    return np.stack([x[i:i + size].mean(axis=0) for i in range(0, x.shape[0], size)])


def select(q: np.ndarray, k: np.ndarray, keep: int, keep_last: int = 0) -> np.ndarray:
    """Lists [query blocks, keep] for one sample and head: q [Tq, d], k [n, d]
    (the sample's own keys); -1 behind the last block."""
    nq = -(-q.shape[0] // QB)
    out = np.full((nq, keep), -1, dtype=np.int32)
    if k.shape[0] == 0:
        return out
    qm, km = _means(q.astype(np.float64), QB), _means(k.astype(np.float64), KB)
    with np.errstate(invalid="ignore"):
        score = np.stack([(row[None] * km).sum(axis=1) for row in qm])     # equal blocks: equal scores
    nk = score.shape[1]
    nan = np.isnan(score)
    score = np.where(nan, -np.inf, score)
    if keep_last:
        score[:, max(0, nk - keep_last):] = np.inf
        nan[:, max(0, nk - keep_last):] = False
    for i in range(nq):
        best = np.sort(np.lexsort((-score[i], nan[i]))[:keep])             # a NaN last, ties in index order
        out[i, :len(best)] = best
    return out


def list_of(entries: Sequence[int], blocks: int) -> list:
    """The blocks a list names: up to its first entry that is not larger than
    the one before, negative, or past the last block."""
    got: list = []
    for e in entries:
        if e < 0 or e >= blocks or (got and e <= got[-1]):
            break
        got.append(int(e))
    return got


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, lists: np.ndarray, scale: Optional[float] = None):
    """(output, sum p |v|, largest sum |q k| scale of a row) for one sample and
    head: q [Tq, d], k and v [n, d], lists [query blocks, keep]."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    scale = 1.0 / np.sqrt(q.shape[1]) if scale is None else scale
    out, mag, top = np.zeros_like(q), np.zeros_like(q), np.zeros((q.shape[0], 1))
    for i in range(lists.shape[0]):
        rows = slice(i * QB, (i + 1) * QB)
        blocks = list_of(lists[i], -(-k.shape[0] // KB))
        if not blocks:
            continue
        at = np.concatenate([np.arange(b * KB, min((b + 1) * KB, k.shape[0])) for b in blocks])
        s = q[rows] @ k[at].T * scale
        p = np.exp(s - s.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        out[rows], mag[rows] = p @ v[at], p @ np.abs(v[at])
        top[rows] = (np.abs(q[rows]) @ np.abs(k[at]).T * scale).max(axis=1, keepdims=True)
    return out, mag, top
