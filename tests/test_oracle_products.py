"""The oracles of the products by kind of row and of the orthogonalised updates, by other means."""
import numpy as np
import pytest

from oracle import products


def setup(comps=1, seed=0):
    rng = np.random.default_rng(seed)
    rows, K, n, ptr = 11, 3, 4, [1, 1, 5, 9]
    return rng.normal(size=(rows, comps * K)), rng.normal(size=(3, K, n)), ptr, rng.permutation(rows), rng.normal(size=(3, n)), rng.normal(size=(rows, comps * n))


@pytest.mark.parametrize("comps", [1, 3])
def test_grouped_row_by_row(comps):
    x, W, ptr, perm, b, _ = setup(comps)
    out = products.grouped(x, W, ptr, perm, b if comps == 1 else None, comps)["out"][0]
    group = {int(perm[p]): g for g in range(3) for p in range(ptr[g], ptr[g + 1])}
    for r in range(x.shape[0]):
        if r not in group:
            assert np.isnan(out[r]).all()
            continue
        for c in range(comps):
            for j in range(4):
                want = sum(x[r, c * 3 + k] * W[group[r], k, j] for k in range(3)) + (b[group[r], j] if comps == 1 else 0)
                assert abs(out[r, c * 4 + j] - want) < 1e-13


@pytest.mark.parametrize("comps", [1, 3])
def test_grouped_gradients_by_differences(comps):
    x, W, ptr, perm, b, t = setup(comps, 1)
    b = b if comps == 1 else None
    r = products.grouped(x, W, ptr, perm, b, comps, t)
    f = lambda x, W, b: np.nansum(products.grouped(x, W, ptr, perm, b, comps)["out"][0] * t)  # noqa: E731
    for name, at in [("gx", 0), ("gW", 1)] + ([("gb", 2)] if comps == 1 else []):
        args = [x, W, b]
        for i in np.ndindex(args[at].shape):
            h = np.zeros(args[at].shape)
            h[i] = 0.5      # the function is linear in each
            up, down = list(args), list(args)
            up[at], down[at] = args[at] + h, args[at] - h
            got = r[name][0][i]
            assert abs((f(*up) - f(*down)) - (0 if np.isnan(got) else got)) < 1e-12, (name, i)


@pytest.mark.parametrize("m,n", [(1, 1), (1, 7), (7, 1), (5, 5), (4, 9), (9, 4)])
def test_orthogonalise_takes_singular_values_through_the_polynomial(m, n):
    G = np.random.default_rng(m * 10 + n).normal(size=(3, m, n))
    out = products.orthogonalise(G, eps=1e-300)
    for g, o in zip(G, out):
        U, s, V = np.linalg.svd(g, full_matrices=False)
        s = s / np.sqrt(np.sum(s ** 2))
        for a, b, c in products.STEPS:
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(o, (U * s) @ V, atol=1e-12)


def test_orthogonalise_of_zeros():
    assert not products.orthogonalise(np.zeros((2, 3, 4))).any()
