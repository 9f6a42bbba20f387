"""The weights' gradients of the gated block over many rows, under bounds by the number of roundings that follow one another.

A sum over rows is formed in splits, each a chain of matrix instructions into the same registers; the splits are joined in eight chains.
A bound that counts the rows themselves would let whole blocks of rows be left out; what these let through is tested as well."""
import numpy as np
import pytest

from oracle import layer
from tests._layer import EPS, check
from tests.test_gpu_gated import inputs, run

UNITS = 256      # compute units

# rows, d_in, d_out: several blocks of 64 rows a split, with narrow and wide outputs, widths of x on both sides of the kernels' borders
SIZES = [(3000, 64, 2176), (2000, 96, 2176), (10_000, 8, 2176), (40_000, 16, 70), (33_000, 100, 97), (20_011, 128, 301), (5000, 37, 1111), (9000, 200, 500), (17_000, 130, 260)]


def roundings(rows, k, n, prec):
    """Roundings one after another in a sum over rows of (weights, biases), and in one over columns of x and of W.

    fp32: an instruction adds 32 products of parts to its registers; six of them make 32 terms.  Each may round (or cut, which is two half
    steps) the registers once; inside it at most 32 roundings of its own 32 products.  fp64: every term rounds once."""
    e, f32 = (4, True) if prec == "f32" else (8, False)
    most = max(1, (64 << 20) // (2 * (k + 1) * n * e))
    if k <= 128:
        alone = k > (64 if f32 else 32)
        groups = 1 if alone else 3 if f32 and k <= 32 else 2
        blocks = -(-rows // 64)
        splits = max(1, min(blocks, groups * UNITS // -(-n // 64), most))
        steps = 2 * -(-blocks // splits)            # of 32 rows
        per_step, pieces = 8, 1
    else:
        piece = min(rows, 8192)
        wide = 64 if f32 else 32
        splits = max(1, min((-(-piece // 32) + 7) // 8, 2 * UNITS // (-(-n // wide) * -(-k // 64)), most))
        steps, per_step, pieces = -(-(-(-piece // 32)) // splits), 8, -(-rows // 8192)
    join = -(-splits // 8) + 4 + pieces
    chain = lambda s: 2 * (6 * s + 34) if f32 else 32 * s  # noqa: E731
    return chain(steps) * (1 if pieces == 1 else pieces) + join, per_step * steps * pieces + 2 + join, chain(-(-k // 32)) + 4, 2 * chain(-(-n // 32)) + 8


def tolerances(ref, rows, k, n, prec):
    w, b, over_k, over_n = roundings(rows, k, n, prec)
    tiny = 1e-37 if prec == "f32" else 1e-300
    out = {}
    for name in ("gx", "gWg", "gWu", "gbg", "gbu"):
        _, mk, mn, mr, m1 = ref[name]
        # 12 roundings for the activation, its derivative and the products behind them
        out[name] = EPS[prec] * (over_k * mk + over_n * mn + (b if name.startswith("gb") else w) * mr + 12 * m1) + tiny
    return out


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_a_block_of_rows_left_out_is_seen(rows, k, n, prec):
    p = inputs(rows, k, n, prec, True, seed=rows)
    tol = tolerances(layer.gated(*p[:5], layer.SILU, p[5]), rows, k, n, prec)
    for first in (0, rows // 2 // 64 * 64, (rows - 64) // 64 * 64):
        part = layer.gated(p[0][first:first + 64], *p[1:5], layer.SILU, p[5][first:first + 64])
        for name in ("gWg", "gWu", "gbg", "gbu"):
            seen = np.abs(part[name][0]) > tol[name]
            assert seen.mean() > 0.5, (name, first, seen.mean())


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_every_row_counts_once(rows, k, n, prec):
    p = inputs(rows, k, n, prec, True, seed=rows)
    ref = layer.gated(*p[:5], layer.SILU, p[5])
    tol = tolerances(ref, rows, k, n, prec)
    for name, got in zip(("gx", "gWg", "gWu", "gbg", "gbu"), run(p, prec, layer.SILU, True)[1:]):
        check(got.cpu().numpy(), ref[name], tol[name], f"{rows}x{k}x{n} {name}")


@pytest.mark.gpu
def test_accuracy_of_the_sigmoid():
    """What the header states: hardware exponential and reciprocal, one unit each (2^-23), the sum's rounding, and t log2(e) rounded once with a
    constant that is off by 0.22 half steps."""
    import torch
    from paper_2501_13986_amd import binding as b
    t = torch.cat([torch.linspace(-86, 90, 200_001), torch.linspace(-2, 2, 20_001), torch.tensor([-200.0, -1000.0, 1000.0])]).cuda()[:, None]
    one, out = torch.ones((1, 1), device="cuda"), torch.empty_like(t)
    b.gated_forward(t, one, torch.zeros_like(one), out, bg=torch.zeros(1, device="cuda"), bu=torch.ones(1, device="cuda"), act=b.ACT_SIGMOID)
    exact = torch.sigmoid(t.double())
    off = (out.double() - exact).abs()
    assert (off <= 2.0 ** -22).all()
    assert (off <= exact * (6 + 1.25 * t.abs().double()) * 2.0 ** -24 + 2.0 ** -125).all()
