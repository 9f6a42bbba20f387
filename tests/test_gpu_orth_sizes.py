"""Orthogonalised updates in fp64 whose squares are not numbers of fp64: on every path the same formula."""
import numpy as np
import pytest

from tests._products import orth_check
from tests.test_gpu_orth import gradients, run

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# one launch, chunks of columns (of either side, joined shares), tiles
SIZES = [(1, 1), (20, 30), (64, 64), (40, 500), (500, 40), (100, 70), (30, 5000), (150, 160), (190, 140)]


@pytest.mark.parametrize("scale,eps", [(1e-200, 1e-250), (1e-157, 1e-300), (1e-305, 2.3e-308), (1e-200, 1e-197), (1e150, 1e-7), (1e200, 1e-7), (1e305, 1.0)])
@pytest.mark.parametrize("m,n", SIZES)
def test_any_size(m, n, scale, eps):
    G = gradients(2, m, n, "f64", seed=m) * scale
    orth_check(run(G, eps=eps), G, "f64", (m, n, scale), eps=eps)


@pytest.mark.parametrize("m,n", SIZES[1:])
def test_zeros_and_numbers_that_are_not_finite_beside_them(m, n):
    G = gradients(4, m, n, "f64", seed=7) * np.array([1e-200, 1e-200, 1e200, 1e200])[:, None, None]
    G[0] = 0
    G[1, m - 1, n - 1], G[2, 0, 0] = np.inf, np.nan
    got = run(G, eps=1e-250)
    assert not got[0].any() and np.isnan(got[1:3]).all()
    orth_check(got[3:], G[3:], "f64", (m, n), eps=1e-250)


@pytest.mark.parametrize("m,n", SIZES[1:])
def test_far_apart_parts(m, n):
    """Rows, or columns, 250 orders of magnitude smaller than the others count as zero beside them."""
    G = gradients(2, m, n, "f64", seed=8)
    G[0, : m // 2] *= 1e-250
    G[1, :, n // 2:] *= 1e-250
    got = run(G * 1e-50, eps=1e-200)
    orth_check(got, G * 1e-50, "f64", (m, n), eps=1e-200)
    assert (np.abs(got[0, : m // 2]) < 1e-200).all() and (np.abs(got[1, :, n // 2:]) < 1e-200).all()
