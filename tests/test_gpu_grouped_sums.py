"""The matrices' and biases' gradients over many rows, under bounds by the number of roundings that follow one another.

A bound that counts the rows themselves lets rows be left out unseen; what these let through is tested as well."""
import numpy as np
import pytest

from oracle import products
from tests._products import EPS, check
from tests.test_gpu_grouped import inputs, run

# rows, d_in, d_out, sizes of the groups
BIASES = [(2500, 64, 64, [2500]), (3000, 24, 40, [1, 0, 2600, 300]), (20_011, 128, 97, [12_000, 17, 7990]), (70_001, 20, 36, [70_000]), (9000, 200, 130, [4000, 4900]), (40_000, 3, 1, [39_000, 999]),
          (5000, 70, 301, [5000])]


def bias_tolerance(entry, prec, rows):
    """Sums in fp64, one after another, and one rounding of the result to the type."""
    return EPS[prec] * np.abs(entry[0]) + EPS["f64"] * rows * entry[1]


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,K,n,sizes", BIASES)
def test_sums_of_biases_are_rounded_once(rows, K, n, sizes, prec):
    for perm in (False, True):
        p = inputs(rows, K, n, sizes, prec, bias=True, perm=perm, seed=rows)
        ref = products.grouped(p["x"], p["W"], p["ptr"], p["perm"], p["b"], 1, p["gout"])
        check(run(p)["gb"].cpu().numpy(), ref["gb"], bias_tolerance(ref["gb"], prec, max(sizes)), f"perm={perm}")


@pytest.mark.gpu
def test_sums_of_biases_whose_rows_are_far_apart():
    """Rows of x lie up to 2^33 bytes apart."""
    import torch
    from paper_2501_13986_amd import binding as b
    rows, ld = 1100, 1 << 21
    p = inputs(rows, 20, 33, [500, 590], "f32", bias=True, perm=True, seed=1)
    x = torch.empty(rows * ld, dtype=torch.float32, device="cuda").as_strided((rows, 20), (ld, 1))
    x.copy_(torch.from_numpy(p["x"]))
    W, gout, ptr, perm = (torch.from_numpy(p[k]).cuda() for k in ("W", "gout", "ptr", "perm"))
    gx, gW, gb = torch.empty(rows, 20, device="cuda"), torch.empty_like(W), torch.empty(2, 33, device="cuda")
    b.grouped_backward(x, W, gout, gx, gW, ptr, gb=gb, perm=perm)
    ref = products.grouped(p["x"], p["W"], p["ptr"], p["perm"], p["b"], 1, p["gout"])
    check(gb.cpu().numpy(), ref["gb"], bias_tolerance(ref["gb"], "f32", 590), "far")


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,K,n,sizes", BIASES)
def test_a_row_left_out_of_a_bias_is_seen(rows, K, n, sizes, prec):
    p = inputs(rows, K, n, sizes, prec, bias=True, seed=rows)
    gout, big = p["gout"].astype(np.float64), int(np.argmax(sizes))
    at = slice(p["ptr"][big], p["ptr"][big + 1])
    tol = bias_tolerance((gout[at].sum(0), np.abs(gout[at]).sum(0)), prec, sizes[big])
    for r in (at.start, (at.start + at.stop) // 2, at.stop - 1):
        assert (np.abs(gout[r]) > 2 * tol).mean() > 0.9
