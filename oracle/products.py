"""Products by kind of row and orthogonalised updates, fp64 numpy.

The products come with the sum of the magnitudes that entered each number: a program that rounds every operation is off by a multiple of
the unit roundoff times that.
"""
from __future__ import annotations

import numpy as np

STEPS = ((3.4445, -4.7750, 2.0315),) * 5


def grouped(x, W, ptr, perm=None, b=None, comps=1, gout=None):
    """A dict of (value, magnitude): out and, given gout, gx, gW, gb.  Rows of no group are NaN in out and gx.  Positions whose perm is outside are left
    out, numbers of ptr outside are taken for the nearest inside."""
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    rows, (groups, K, n) = x.shape[0], W.shape
    perm = np.arange(rows) if perm is None else np.asarray(perm)
    ptr = np.clip(np.asarray(ptr), 0, rows)
    x3 = x.reshape(rows, comps, K)
    out, m_out = np.full((rows, comps, n), np.nan), np.zeros((rows, comps, n))
    gx, m_gx = np.full((rows, comps, K), np.nan), np.zeros((rows, comps, K))
    gW, m_gW, gb, m_gb = np.zeros(W.shape), np.zeros(W.shape), np.zeros((groups, n)), np.zeros((groups, n))
    for g in range(groups):
        at = perm[ptr[g]:ptr[g + 1]]
        at = at[(at >= 0) & (at < rows)]
        if at.size == 0:
            continue
        add = np.zeros(n) if b is None else np.asarray(b[g], np.float64)
        out[at], m_out[at] = x3[at] @ W[g] + add, np.abs(x3[at]) @ np.abs(W[g]) + np.abs(add)
        if gout is not None:
            t = np.asarray(gout, np.float64).reshape(rows, comps, n)[at]
            gx[at], m_gx[at] = t @ W[g].T, np.abs(t) @ np.abs(W[g]).T
            flat_x, flat_t = x3[at].reshape(-1, K), t.reshape(-1, n)
            gW[g], m_gW[g] = flat_x.T @ flat_t, np.abs(flat_x).T @ np.abs(flat_t)
            gb[g], m_gb[g] = flat_t.sum(0), np.abs(flat_t).sum(0)
    back = {"out": (out.reshape(rows, -1), m_out.reshape(rows, -1))}
    if gout is not None:
        back.update(gx=(gx.reshape(rows, -1), m_gx.reshape(rows, -1)), gW=(gW, m_gW), gb=(gb, m_gb))
    return back


def orthogonalise(G, coefficients=STEPS, eps=1e-7, dtype=np.float64):
    """Of each matrix of a batch; dtype: what every step is rounded to (the sum of squares is held in 64 bits)."""
    G = np.asarray(G)
    out = np.empty(G.shape, dtype)
    for i, g in enumerate(G):
        X = (g.astype(np.longdouble) / (np.sqrt(np.sum(g.astype(np.longdouble) ** 2)) + eps)).astype(dtype)
        X = X if X.shape[0] <= X.shape[1] else X.T.copy()
        for a, b, c in coefficients:
            A = X @ X.T
            X = dtype(a) * X + (dtype(b) * A + dtype(c) * (A @ A)) @ X
        out[i] = X if g.shape[0] <= g.shape[1] else X.T
    return out
