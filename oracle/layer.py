"""The layer operators around the convolution, fp64 numpy: gated feed-forward block and group normalisation of irreps rows.

Every function returns its result and, in the same layout, the sum of the magnitudes that entered each number: a program that
rounds every operation is off by a multiple of the unit roundoff times that.
"""
from __future__ import annotations

from math import erf, pi, sqrt

import numpy as np

from .irreps import parse_irreps

NONE, SILU, GELU, SIGMOID, TANH = range(5)


def act(t, kind):
    """act(t), act'(t)."""
    t = np.asarray(t, dtype=np.float64)
    with np.errstate(over="ignore"):
        q = 1.0 / (1.0 + np.exp(-t))
    if kind == SILU:
        return t * q, q * (1 + t * (1 - q))
    if kind == GELU:
        p = 0.5 * (1 + np.vectorize(erf, otypes=[float])(t / sqrt(2.0)))
        return t * p, p + t * np.exp(-t * t / 2) / sqrt(2 * pi)
    if kind == SIGMOID:
        return q, q * (1 - q)
    if kind == TANH:
        return np.tanh(t), 1 - np.tanh(t) ** 2
    return t, np.ones_like(t)


# ---- gated feed-forward block -------------------------------------------------------------------------------------------

def gated(x, Wg, Wu, bg, bu, kind, gout=None):
    """(out, gx, gWg, gWu, gbg, gbu) and the magnitudes of each, in units of `terms` roundings of a projection's sum: a dict
    name -> (value, roundings of sums over d_in, of sums over d_out, of sums over rows, single roundings)."""
    x, Wg, Wu = (np.asarray(a, np.float64) for a in (x, Wg, Wu))
    bg = np.zeros(Wg.shape[1]) if bg is None else np.asarray(bg, np.float64)
    bu = np.zeros(Wg.shape[1]) if bu is None else np.asarray(bu, np.float64)
    g, u = x @ Wg + bg, x @ Wu + bu
    G, U = np.abs(x) @ np.abs(Wg) + np.abs(bg), np.abs(x) @ np.abs(Wu) + np.abs(bu)
    a, d = act(g, kind)
    out = {"out": (a * u, 1.13 * np.abs(u) * G + np.abs(a) * U, 0, 0, (np.abs(a) + 1) * np.abs(u))}
    if gout is None:
        return out
    t = np.asarray(gout, np.float64)
    dg, du = t * u * d, t * a
    # |act'| <= 1.13, |act''| <= 1: what an error of the projections does to dg and du, and single roundings
    dgK, duK = np.abs(t) * (np.abs(u) * G + 1.13 * U), np.abs(t) * 1.13 * G
    dg1, du1 = np.abs(t) * np.abs(u) * 1.13, np.abs(t) * (np.abs(a) + 1)
    aWg, aWu, ax = np.abs(Wg), np.abs(Wu), np.abs(x)
    out["gx"] = (dg @ Wg.T + du @ Wu.T, dgK @ aWg.T + duK @ aWu.T, np.abs(dg) @ aWg.T + np.abs(du) @ aWu.T, 0, dg1 @ aWg.T + du1 @ aWu.T)
    out["gWg"] = (x.T @ dg, ax.T @ dgK, 0, ax.T @ np.abs(dg), ax.T @ dg1)
    out["gWu"] = (x.T @ du, ax.T @ duK, 0, ax.T @ np.abs(du), ax.T @ du1)
    out["gbg"] = (dg.sum(0), dgK.sum(0), 0, np.abs(dg).sum(0), dg1.sum(0))
    out["gbu"] = (du.sum(0), duK.sum(0), 0, np.abs(du).sum(0), du1.sum(0))
    return out


# ---- group normalisation ------------------------------------------------------------------------------------------------

def norm_segments(irreps, gated_):
    """(mul, components, invariant, first column of x, of y, first column of the gates or -1)."""
    out, at = [], 0
    for ir in parse_irreps(irreps):
        out.append([ir.mul, 2 * ir.l + 1, ir.l == 0 and ir.p > 0, at, at, -1])
        at += ir.mul * (2 * ir.l + 1)
    dim_y = at
    if gated_:
        for s in out:
            if not s[2]:
                s[5] = at
                at += s[0]
    return out, at, dim_y


def norm(irreps, groups, kind, gated_, eps, ir_mul, x, weight, bias, ptr=None, gy=None):
    """A dict: y, stats [S, segments, groups, 2] and, given gy, gx, gweight, gbias; each (value, magnitude).  Rows of no sample are
    NaN in y and gx.  ptr None: every row a sample."""
    segs, dim_x, dim_y = norm_segments(irreps, gated_)
    x, weight, bias = (np.asarray(a, np.float64) for a in (x, weight, bias))
    N = x.shape[0]
    ptr = list(range(N + 1)) if ptr is None else [int(p) for p in ptr]
    S, n_gate = len(ptr) - 1, sum(s[5] >= 0 for s in segs)
    y, gx = np.full((N, dim_y), np.nan), np.full((N, dim_x), np.nan)
    my, mx = np.zeros((N, dim_y)), np.zeros((N, dim_x))
    stats, mstats = np.zeros((S, len(segs) + n_gate, groups, 2)), np.zeros((S, len(segs) + n_gate, groups, 2))
    gw, mw, gb, mb = np.zeros(weight.size), np.zeros(weight.size), np.zeros(bias.size), np.zeros(bias.size)
    ws, at = [], 0
    for s in segs:
        ws.append(at)
        at += s[0]
    bs, bt = [], 0
    for s in segs:
        bs.append(bt if s[2] else -1)
        bt += s[0] if s[2] else 0
    gate_ws, gate_bs = [], []
    for s in segs:
        gate_ws.append(at)
        gate_bs.append(bt)
        if s[5] >= 0:
            at, bt = at + s[0], bt + s[0]

    def columns(first, mul, n, g):
        ch = np.arange(g * (mul // groups), (g + 1) * (mul // groups))
        comp = np.arange(n)
        return first + (comp[None, :] * mul + ch[:, None] if ir_mul else ch[:, None] * n + comp[None, :]), ch

    def unit(v, inv):
        """xh, mu, r, and the magnitude of an error of xh in units of the roundoff."""
        if v.size == 0:
            return v, 0.0, 1 / sqrt(eps), np.zeros_like(v), 0.0
        mu = v.mean() if inv else 0.0
        r = 1 / sqrt(((v - mu) ** 2).mean() + eps)
        mean = np.abs(v).mean() if inv else 0.0
        return (v - mu) * r, mu, r, r * (mean + np.abs(v - mu)), mean

    for i in range(S):
        rows = np.arange(ptr[i], max(ptr[i], ptr[i + 1]))
        place = len(segs)
        for k, (mul, n, inv, col, ycol, gate) in enumerate(segs):
            for g in range(groups):
                cols, ch = columns(col, mul, n, g)
                ycols = cols - col + ycol
                v = x[np.ix_(rows, cols.ravel())].reshape(len(rows), len(ch), n)
                xh, mu, r, ex, mean = unit(v, inv)
                stats[i, k, g], mstats[i, k, g] = (mu, r), (mean, r)
                w = weight[ws[k] + ch][None, :, None]
                q, sens = 1.0, 0.0
                if gate >= 0:
                    gcols, _ = columns(gate, mul, 1, g)
                    gv = x[np.ix_(rows, gcols.ravel())].reshape(len(rows), len(ch), 1)
                    gh, gmu, gr, egx, gmean = unit(gv, True)
                    stats[i, place, g], mstats[i, place, g] = (gmu, gr), (gmean, gr)
                    wg, bgate = weight[gate_ws[k] + ch][None, :, None], bias[gate_bs[k] + ch][None, :, None]
                    lg = wg * gh + bgate
                    q = 1 / (1 + np.exp(-lg))
                    elg = np.abs(wg) * egx + np.abs(lg) + np.abs(bgate) + 1
                if inv:
                    lin = w * xh + bias[bs[k] + ch][None, :, None]
                    elin = np.abs(w) * ex + np.abs(lin) + np.abs(w * xh)
                    a, d = act(lin, kind)
                    yv, ey = a, 1.13 * elin + np.abs(a) + 1
                else:
                    lin = w * xh
                    elin = np.abs(w) * ex + np.abs(lin)
                    yv, ey = lin * q, elin + (np.abs(lin) * elg if gate >= 0 else 0)
                y[np.ix_(rows, ycols.ravel())] = yv.reshape(len(rows), cols.size)
                my[np.ix_(rows, ycols.ravel())] = ey.reshape(len(rows), cols.size)
                if gy is None:
                    continue
                t = np.asarray(gy, np.float64)[np.ix_(rows, ycols.ravel())].reshape(len(rows), len(ch), n)
                if inv:
                    l, el = t * d, np.abs(t) * (elin + 1.13)
                else:
                    l, el = t * q, np.abs(t) * ((elg if gate >= 0 else 0) + 1)

                def back(l, el, xh, ex, r, w, inv, at_w, at_b, cols):
                    h, eh, M = l * w, el * np.abs(w), l.size
                    gw[at_w + ch] += (l * xh).sum((0, 2))
                    mw[at_w + ch] += (el * np.abs(xh) + np.abs(l) * ex + np.abs(l * xh)).sum((0, 2))
                    if inv:
                        gb[at_b + ch] += l.sum((0, 2))
                        mb[at_b + ch] += (el + np.abs(l)).sum((0, 2))
                    if M == 0:
                        return
                    m1, m2 = h.mean() if inv else 0.0, (h * xh).mean()
                    e1 = (eh + np.abs(h)).mean() if inv else 0.0
                    e2 = (eh * np.abs(xh) + np.abs(h) * ex + np.abs(h * xh)).mean()
                    gx[np.ix_(rows, cols.ravel())] = (r * (h - m1 - xh * m2)).reshape(len(rows), cols.size)
                    e = r * (eh + np.abs(h) + e1 + np.abs(m1) + np.abs(xh) * e2 + (ex + np.abs(xh)) * np.abs(m2))
                    mx[np.ix_(rows, cols.ravel())] = e.reshape(len(rows), cols.size)

                back(l, el, xh, ex, r, w, inv, ws[k], bs[k], cols)
                if gate >= 0:
                    s = (t * lin).sum(2, keepdims=True)
                    ms = (np.abs(t) * (elin + np.abs(lin))).sum(2, keepdims=True)
                    lg_, elg_ = s * q * (1 - q), 0.25 * ms + np.abs(s) * elg
                    back(lg_, elg_, gh, egx, gr, wg, True, gate_ws[k], gate_bs[k], gcols)
            if gate >= 0:
                place += 1
    out = {"y": (y, my), "stats": (stats, mstats)}
    if gy is not None:
        out.update(gx=(gx, mx), gweight=(gw, mw), gbias=(gb, mb))
    return out
