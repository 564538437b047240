"""What the tests of attention_masked and of the cache's attention share: the
tolerance of one head's outputs.

With A = sum p |v| per output and u = 2^-24.  A score is off by E at most: its product
by (d + 3) u sum |q k| scale, the distance's share, the change to log2 units and the
exponent's difference by 8u of its size, a capped one also by 4u of the cap (bf16: by
2^-22 of it, caps to 1000, beyond by 2^-20 of the score).  A probability is off by E of
itself, and so is their sum: 2 E A.  bf16: the probabilities are rounded (2^-8 A), the
row sums are those of the rounded ones (2^-8 A again), the output is rounded (2^-8 of
itself); sums and the exponential are below 2 % of that.  fp32: sums of n terms, n u A,
and 20 u A for the rest."""
import numpy as np

U = 2.0 ** -24


def tolerance(want, A, size, mag, d, n, cap, bf16):
    E = (d + 3) * U * size + 8 * U * mag
    if cap:
        E = E + (4 * U * cap if not bf16 else 2.0 ** -22 * cap if cap <= 1000 else 2.0 ** -20 * mag)
    tol = 2 * E[:, None] * A
    with np.errstate(invalid="ignore"):
        if bf16:
            return tol + 2.0 ** -8 * 1.02 * (2 * A + np.abs(want)) + 1e-30
        return tol + (n + 20) * U * A + 1e-30


def compare(got, want, tol, A):
    """Finite outputs within the tolerance; the others are the formula's infinities and NaN."""
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    err = np.abs(got[fin] - want[fin])
    assert np.all(err <= tol[fin]), float((err / tol[fin]).max())
    none = (A == 0).all(1)
    assert not got[none].any()
