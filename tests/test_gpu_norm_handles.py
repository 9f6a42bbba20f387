"""The normalisation of every kind of handle against the fp64 oracle: groups that registers do not hold."""
import pytest

from oracle import layer
from tests._layer import check, norm_tolerance
from tests.test_gpu_norm import GRAPHS, IRREPS, LARGE, compare, handle, inputs, run, torch
from tests.test_layer_handles import MANY, WIDE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("ir_mul", [False, True])
@pytest.mark.parametrize("irreps", WIDE)
def test_wide_groups(irreps, ir_mul, prec):
    for act, gated in ((layer.SILU, True), (layer.TANH, False)):
        n = handle(irreps, 1, act, gated, prec, ir_mul)
        for ptr in (None, [0, 5, 5, 11], [2, 12]):
            p = inputs(n, 12, prec, seed=3)
            compare(run(n, p, ptr), irreps, 1, act, gated, ir_mul, p, prec, ptr)


def test_many_segments():
    n = handle(MANY, 1, layer.NONE, True, "f32", False)
    for ptr in (None, [0, 2, 2, 7]):
        p = inputs(n, 7, "f32", seed=1)
        compare(run(n, p, ptr), MANY, 1, layer.NONE, True, False, p, "f32", ptr)


# one of the four calls at least is served by the kernels for any size, the others by registers
MIXED = [("512x0e+512x1o", 1), ("2048x0e", 1), ("1536x0e", 1), ("256x0e+256x1o+256x2e+256x3o", 1), ("1024x0e", 1)]


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("irreps,groups", MIXED)
def test_calls_with_kernels_of_both_kinds(irreps, groups, prec):
    """Forward and backward exchange statistics and nothing else; samples longer than a chunk among them."""
    n = handle(irreps, groups, layer.SILU, True, prec, False)
    for N, ptr in ((5, None), (300, [0, 300]), (290, [0, 3, 3, 40, 200, 287])):
        p = inputs(n, N, prec, seed=N)
        compare(run(n, p, ptr), irreps, groups, layer.SILU, True, False, p, prec, ptr)


# scalar registers that went to a vector register's lanes leave room for private memory that nothing uses
ROOM = [("48x0e+10x1o+10x1e+48x0o", 1), ("7x0e+5x1o+3x2e+9x0e", 1), ("32x0e+32x1o+32x2e+32x3o", 1), ("4x0e+4x1o+4x1e+4x2e", 4)]


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("irreps,groups", ROOM)
def test_code_with_unused_private_room(irreps, groups, prec):
    n = handle(irreps, groups, layer.NONE, True, prec, True)
    for N, ptr in ((7, None), (1000, [0, 1000]), (900, [0, 2, 2, 60, 500, 899])):
        p = inputs(n, N, prec, seed=N)
        compare(run(n, p, ptr), irreps, groups, layer.NONE, True, True, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("irreps,groups,N", [("300x8e", 1, 2600), ("700x0e+512x3o", 1, 2300), ("96x7o", 1, 2500), ("260x6e", 2, 1300)])
def test_more_samples_than_rows_of_partial_sums(irreps, groups, N, prec):
    """A workgroup has several samples, some without rows, also the first."""
    n = handle(irreps, groups, layer.SILU, True, prec, False)
    if irreps == "300x8e":      # over the limit of words; the others are held in registers or not as the compiler has it
        assert n.kernel(True, True) == n.kernel(False, True) == "cgtp_norm_unit_bwd"
    p = inputs(n, N, prec, seed=N)
    wide = [a.astype("float64") for a in p]
    ends = sorted([0, 0, 0, 1, 1, N] + [min(N, 2 * i // 3) for i in range(N)])
    for ptr in (None, ends):
        got = run(n, p, ptr)
        compare(got, irreps, groups, layer.SILU, True, False, wide, prec, ptr)
        again = run(n, p, ptr)
        for k in got:
            assert torch.equal(torch.nan_to_num(got[k]), torch.nan_to_num(again[k])), k


def test_cost_of_a_long_sample_grows_with_its_rows():
    """Eight times the rows of one sample in 32 groups take eight times as long; when every chunk summed up all the others it was 33 times."""
    from paper_2501_13986_amd import binding as b
    n = handle("128x0e", 32, layer.SILU, True, "f32", False)

    def time(N):
        x, w, bias = torch.randn((N, n.dim_x), device="cuda"), torch.ones(n.n_w, device="cuda"), torch.zeros(n.n_b, device="cuda")
        y, stats, ptr = torch.empty((N, n.dim_y), device="cuda"), torch.empty(n.n_stat, device="cuda"), torch.tensor([0, N], device="cuda")
        gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(bias)
        best = float("inf")
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            b.norm_forward(n, x, w, bias, y, stats, ptr=ptr)
            b.norm_backward(n, x, w, bias, x, stats, gx, gw, gb, ptr=ptr)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        return best

    assert time(1_000_000) < 16 * time(125_000)


@pytest.mark.parametrize("ends", [[0, 150_000], [5, 90_000, 90_001, 90_040, 149_990]])
def test_samples_of_many_chunks(ends):
    """Chunks of more than 128 rows, several of them and several samples a workgroup."""
    irreps = "8x0e+4x1o"
    n = handle(irreps, 2, layer.SILU, True, "f32", False)
    p = inputs(n, 150_000, "f32", seed=3)
    compare(run(n, p, ends), irreps, 2, layer.SILU, True, False, [a.astype("float64") for a in p], "f32", ends)


@pytest.mark.parametrize("row", [0, 10_000, 19_999])
def test_a_number_far_from_all_others(row):
    """fp64: wherever it stands, the variance has its digits.  Sums about a number of the sample's bulk have no cancellation beyond that of
    their terms, of which at most 400 are added one after another (a wave's rows of a chunk, waves, the chunks' shares)."""
    irreps, N = "8x0e+8x1o", 20_000
    n = handle(irreps, 1, layer.NONE, True, "f64", False)
    p = inputs(n, N, "f64", seed=7, shift=3.0, scale=1.0)
    p[0][row, 0], p[0][row, n.dim_y] = 1e8, -1e9      # of the scalars and of the gates
    ref = layer.norm(irreps, 1, layer.NONE, True, 1e-5, False, *p[:3], [0, N])
    got = run(n, p, [0, N])
    for k in ("stats", "y"):
        check(got[k].cpu().numpy().reshape(ref[k][0].shape), ref[k], norm_tolerance(ref[k], "f64", 400), k)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("ir_mul", [False, True])
@pytest.mark.parametrize("irreps,groups", IRREPS + LARGE)
def test_without_gates(irreps, groups, ir_mul, prec):
    n = handle(irreps, groups, layer.SILU, False, prec, ir_mul)
    for i, ptr in enumerate(GRAPHS):
        p = inputs(n, 41 if ptr is not None else 37, prec, seed=i)
        compare(run(n, p, ptr), irreps, groups, layer.SILU, False, ir_mul, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", [layer.NONE, layer.GELU, layer.SIGMOID, layer.TANH])
def test_activations_in_the_other_layout(act, gated, prec):
    irreps = "12x0e+4x1o"
    n = handle(irreps, 2, act, gated, prec, True)
    for ptr in (None, [0, 9, 20]):
        p = inputs(n, 20, prec, seed=act)
        compare(run(n, p, ptr), irreps, 2, act, gated, True, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("irreps,groups", [("32x0e+32x1o", 4), ("512x0e+512x1o", 1)])
def test_runs_are_bit_identical_and_finite(irreps, groups, prec):
    n = handle(irreps, groups, layer.SILU, True, prec, False)
    p = inputs(n, 4000, prec)
    for ptr in (None, [0, 4000], [0, 5, 1200, 4000]):
        a, c = run(n, p, ptr), run(n, p, ptr)
        for k in a:
            assert torch.isfinite(a[k]).all() and torch.equal(a[k], c[k]), k
