"""Tolerances of the layer operators, from the magnitudes that oracle.layer returns."""
import numpy as np

EPS = {"f32": 2.0 ** -24, "f64": 2.0 ** -53}   # half a step


def gated_tolerance(entry, prec, k, n, rows):
    """A projection's sum over d_in has k terms; in fp32 every product is six of bf16 parts, each added with one rounding at
    most, and what the parts leave out (2^-25) is less than one more.  The gradients' sums have 2 n terms (both projections) and
    `rows` terms in the same way.  16: the start, the bias, joins of partial sums.  12 roundings for the activation, its derivative
    and the products behind them."""
    _, mk, mn, mr, m1 = entry
    p = 6 if prec == "f32" else 1
    tiny = 1e-37 if prec == "f32" else 1e-300    # results below the normal numbers
    return EPS[prec] * ((p * k + 16) * mk + (2 * p * n + 16) * mn + (p * rows + 16) * mr + 12 * m1) + tiny


def norm_tolerance(entry, prec, count):
    """64 roundings of the magnitudes.  fp32 sums are held in 64 bits, or are trees over a row's lanes with at most 40 terms one
    after another; fp64 sums round once for each of `count` terms."""
    return EPS[prec] * (64 + (count if prec == "f64" else 0)) * entry[1] + (1e-37 if prec == "f32" else 1e-300)


def check(got, entry, tol, what):
    got, ref = np.asarray(got, np.float64), entry[0]
    assert got.shape == np.shape(ref), (what, got.shape, np.shape(ref))
    assert np.all(np.isfinite(got)), f"{what}: non-finite values"
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]}, tolerance {np.broadcast_to(tol, bad.shape)[bad][0]}"
