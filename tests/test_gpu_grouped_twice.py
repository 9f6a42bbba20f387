"""Rows that a permutation names twice: each number is that of one of their positions, and both count in the matrices' gradients."""
import numpy as np
import pytest

from oracle import products
from tests._products import check, grouped_tolerance
from tests.test_gpu_grouped import inputs, run

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("K,n", [(16, 300), (300, 16), (140, 150), (16, 20)])
def test_each_number_is_that_of_one_position(K, n, prec):
    rows, cut = 150, 80
    p = inputs(rows, K, n, [cut, rows - cut], prec, bias=True, perm=True, seed=K)
    twice = [(100, 10), (120, 40), (5, 6)]      # positions of both groups, of both groups, of one
    for to, of in twice:
        p["perm"][to] = p["perm"][of]
    o = run(p)
    named = np.zeros(rows, bool)
    named[p["perm"]] = True
    at = p["perm"]
    for name, terms in (("out", K), ("gx", n)):
        got = o[name].cpu().numpy().astype(np.float64)
        assert np.isnan(got[~named]).all()
        left = np.ones(got.shape, bool)
        for g, positions in enumerate((slice(0, cut), slice(cut, rows))):      # as if all rows were of this group: the oracle's number for them there
            ref = products.grouped(p["x"], p["W"][g:g + 1], [0, rows], None, p["b"][g:g + 1], 1, p["gout"])[name]
            mine = np.zeros(rows, bool)
            mine[at[positions]] = True
            left &= ~(mine[:, None] & (np.abs(got - ref[0]) <= grouped_tolerance(ref, prec, terms)))
        assert not left[named].any()
    for g, positions in enumerate((slice(0, cut), slice(cut, rows))):
        x, t = p["x"][at[positions]].astype(np.float64), p["gout"][at[positions]].astype(np.float64)
        for name, ref in (("gW", (x.T @ t, np.abs(x).T @ np.abs(t))), ("gb", (t.sum(0), np.abs(t).sum(0)))):
            check(o[name][g].cpu().numpy(), ref, grouped_tolerance(ref, prec, rows), f"{name} {g}")
