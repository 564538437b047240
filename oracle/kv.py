"""What a key-value cache in 8 bits holds, in float64 (every value is exact)."""
from __future__ import annotations

import numpy as np

BLOCK = 64


def scale_of(x: np.ndarray) -> float:
    """The least power of two from 2^-100 up with max|x| <= 448 times it (what is not finite left aside)."""
    x = np.abs(x[np.isfinite(x)])
    s = 2.0 ** -100
    while x.size and x.max() > 448.0 * s:
        s *= 2.0
    return s


def round8(y: np.ndarray) -> np.ndarray:
    """To nearest in e4m3, ties to even; what is not finite to NaN."""
    y = np.asarray(y, np.float64)
    fin = np.isfinite(y)
    z = np.where(fin, y, 0.0)
    step = 2.0 ** (np.maximum(np.frexp(z)[1] - 1, -6) - 3)
    return np.where(fin, np.rint(z / step) * step, np.nan)


class Cache:
    """One of keys and values: [B][H] of `capacity` tokens."""

    def __init__(self, B: int, H: int, d: int, capacity: int):
        self.val = np.zeros((B, H, capacity, d))
        self.scale = np.zeros((B, H, -(-capacity // BLOCK)))
        self.capacity = capacity

    def push(self, x: np.ndarray, lens, counts):
        """x [B, T, H, d]: sample b's first counts[b] tokens end at lens[b]."""
        for b in range(x.shape[0]):
            n, c = min(max(int(lens[b]), 0), self.capacity), min(max(int(counts[b]), 0), x.shape[1])
            at = np.arange(n - c, n)
            new, at = x[b, :c][at >= 0], at[at >= 0]
            for blk in np.unique(at // BLOCK):
                rows = at[at // BLOCK == blk]
                for h in range(x.shape[2]):
                    y = new[at // BLOCK == blk, h].astype(np.float64)
                    s, held = scale_of(y), slice(blk * BLOCK, rows[0])
                    if rows[0] > blk * BLOCK:
                        s = max(s, self.scale[b, h, blk])
                        self.val[b, h, held] = round8(self.val[b, h, held] / s) * s
                    self.val[b, h, rows] = round8(y / s) * s
                    self.scale[b, h, blk] = s
