"""Rotary positions in float64."""
from __future__ import annotations

import math
from typing import Sequence

import numpy as np


def frequencies(n: int, theta: float, scaling: str = "none", factor: float = 1.0, original: int = 0,
                beta_fast: float = 32.0, beta_slow: float = 1.0) -> np.ndarray:
    """Radians per position of the n / 2 pairs of an axis of n columns."""
    out = []
    for j in range(n // 2):
        base = theta * factor ** (n / (n - 2)) if scaling == "ntk" and n > 2 else theta
        f = math.exp(-2.0 * j / n * math.log(base))
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            turns = original * f / (2 * math.pi)
            if turns <= beta_slow:
                f /= factor
            elif turns < beta_fast:
                share = (turns - beta_slow) / (beta_fast - beta_slow)
                f = share * f + (1 - share) * f / factor
        out.append(f)
    return np.array(out)


def turn(x: np.ndarray, pos: np.ndarray, axes: Sequence[int], freqs: np.ndarray, layout: str, amplitude: float = 1.0,
         inverse: bool = False) -> np.ndarray:
    """x [B, T, H, d] with the leading sum(axes) columns of each head turned; pos [B, T, len(axes)]."""
    out = x.astype(np.float64).copy()
    col = pair = 0
    for axis, n in enumerate(axes):
        for j in range(n // 2):
            a, b = (col + 2 * j, col + 2 * j + 1) if layout == "pairs" else (col + j, col + n // 2 + j)
            phi = pos[..., axis].astype(np.float64) * freqs[pair + j]
            c, s = amplitude * np.cos(phi)[..., None], amplitude * np.sin(phi)[..., None]
            if inverse:
                s = -s
            xa, xb = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
            out[..., a], out[..., b] = xa * c - xb * s, xa * s + xb * c
        col += n
        pair += n // 2
    return out
