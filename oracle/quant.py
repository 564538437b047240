"""Quantised cache slots: what a feature reads back as.

Groups of 64 consecutive values of the flat feature share the scale
s = fl32(max|x| / Q), Q = 127 for 8 bits and 7 for 4; a value is held as
x / s rounded to the nearest integer (ties to even).  A scale below 2^-120 is
zero; a group with a value that is not finite reads back as NaN.
"""
from __future__ import annotations

import numpy as np

GROUP = 64
MIN_SCALE = 2.0 ** -120


def codes(x: np.ndarray, bits: int):
    """(codes [groups, 64], scales [groups, 1]) in float64, of float32 values
    (bfloat16 ones among them)."""
    q = {8: 127.0, 4: 7.0}[bits]
    flat = np.asarray(x, dtype=np.float64).ravel()
    g = np.zeros(-(-flat.size // GROUP) * GROUP)
    g[:flat.size] = flat
    g = g.reshape(-1, GROUP)
    top = np.abs(g).max(axis=1, keepdims=True)
    bad = ~np.isfinite(top)
    with np.errstate(invalid="ignore"):
        # The division in float64, then one rounding to float32, is the correctly
        # rounded float32 division (53 >= 2 * 24 + 2).
        s = np.where(bad, 1.0, top / q).astype(np.float32).astype(np.float64)
        s[s < MIN_SCALE] = 0.0
        n = np.where(s > 0, np.rint(g / np.where(s > 0, s, 1.0)), 0.0)
    return np.where(bad, 0.0, n), np.where(bad, np.nan, s)


def held(x: np.ndarray, bits: int) -> np.ndarray:
    """The values that a slot holding x stands for, in float64, x's shape."""
    n, s = codes(x, bits)
    return (n * s).ravel()[:np.asarray(x).size].reshape(np.shape(x))
