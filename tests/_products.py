"""Tolerances of the products by kind of row and of the orthogonalised updates."""
import numpy as np

from oracle import products

EPS = {"f32": 2.0 ** -24, "f64": 2.0 ** -53}   # half a step


def grouped_tolerance(entry, prec, terms):
    """A sum of `terms` products: in fp32 each is six of bf16 parts, each added with one rounding at most, and what the parts leave out (2^-25)
    is less than one more.  16: the start, the bias, joins of partial sums."""
    return EPS[prec] * ((6 if prec == "f32" else 1) * terms + 16) * entry[1] + (1e-37 if prec == "f32" else 1e-300)


def check(got, entry, tol, what):
    """Rows of no group are NaN in the oracle and have to be what they were: NaN here."""
    got, ref = np.asarray(got, np.float64), entry[0]
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: other rows are written than those of groups"
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]}, tolerance {np.broadcast_to(tol, bad.shape)[bad][0]}"


def orth_check(got, G, prec, what, coefficients=products.STEPS, eps=1e-7):
    """Against the steps in a longer type, by the size (root of the sum of squares) of the difference in each matrix.  The bound is computed, not chosen:
    the steps take a rounding along as they take the singular values, up to 3.4 times a step, so the same formulas are run with every matrix
    rounded to the type, products summed as the CPU's library does, and their difference is the measure of what roundings do to this
    matrix.  8 times that: a kernel rounds six products of parts for one (a random walk of sqrt 6 times the steps: 2.5) and may sum one term after
    another where the library has 8 to 16 chains (a walk 3 times longer); and 32 roundings of numbers of a size of at most 1.3 sqrt(s)."""
    long_, short = (np.float64, np.float32) if prec == "f32" else (np.longdouble, np.float64)
    got = np.asarray(got)
    ref, same = products.orthogonalise(G, coefficients, eps, long_), products.orthogonalise(G, coefficients, eps, short)
    size = lambda v: np.sqrt(np.sum(v.astype(np.longdouble) ** 2, (1, 2)))  # noqa: E731
    off, tol = size(got - ref), 8 * size(same - ref) + 32 * EPS[prec] * size(ref)
    assert np.all(np.isfinite(got)) and np.all(off <= tol), f"{what}: matrix {int(np.argmax(off - tol))}: {off.max()} for {tol[np.argmax(off - tol)]}"
