"""The group normalisation of irreps rows against the fp64 oracle."""
import numpy as np
import pytest

from oracle import layer
from tests._layer import check, norm_tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def handle(irreps, groups, act, gated, prec, ir_mul, eps=1e-5):
    from paper_2501_13986_amd import binding as b
    return b.Norm(irreps, groups=groups, act=act, gated=gated, eps=eps, dtype=b.CGTP_F64 if prec == "f64" else b.CGTP_F32, device=0,
                  flags=b.CGTP_IR_MUL if ir_mul else b.CGTP_MUL_IR)


def inputs(n, N, prec, seed=0, shift=1.0, scale=2.0):
    rng = np.random.default_rng(seed)
    p = [rng.normal(size=(N, n.dim_x)) * scale + shift, 1 + 0.3 * rng.normal(size=n.n_w), 0.3 * rng.normal(size=n.n_b), rng.normal(size=(N, n.dim_y))]
    return [a.astype(np.float32 if prec == "f32" else np.float64) for a in p]


def run(n, p, ptr=None, fill=float("nan")):
    from paper_2501_13986_amd import binding as b
    x, w, bias, gy = [torch.from_numpy(a).cuda() for a in p]
    N = x.shape[0]
    t = None if ptr is None else torch.tensor(ptr, dtype=torch.int64, device="cuda")
    S = N if ptr is None else len(ptr) - 1
    new = lambda *s: torch.full(s, fill, dtype=x.dtype, device="cuda")  # noqa: E731
    y, stats, gx, gw, gb = new(N, n.dim_y), new(S, n.n_stat), new(N, n.dim_x), new(n.n_w), new(n.n_b)
    b.norm_forward(n, x, w, bias, y, stats, ptr=t)
    b.norm_backward(n, x, w, bias, gy, stats, gx, gw, gb, ptr=t)
    torch.cuda.synchronize()
    return dict(y=y, stats=stats, gx=gx, gweight=gw, gbias=gb)


def compare(got, irreps, groups, act, gated, ir_mul, p, prec, ptr, eps=1e-5):
    ref = layer.norm(irreps, groups, act, gated, eps, ir_mul, p[0], p[1], p[2], ptr, p[3])
    N = p[0].shape[0]
    longest = 1 if ptr is None else max([1] + [e - s for s, e in zip(ptr, ptr[1:])])
    count = longest * p[0].shape[1] // groups
    for name, t in got.items():
        v, tol = t.cpu().numpy().reshape(ref[name][0].shape), norm_tolerance(ref[name], prec, count if name != "gweight" and name != "gbias" else count + N)
        own = ~np.isnan(ref[name][0])
        assert np.isnan(v[~own]).all(), f"{name}: rows of no sample were written"
        check(np.where(own, v, 0), (np.where(own, ref[name][0], 0),), np.where(own, tol, 1), name)


IRREPS = [("32x0e+32x1o+32x2e+32x3o", 4), ("7x0e+5x1o+3x2e+9x0e", 1), ("48x0e+10x1o+10x1e+48x0o", 2), ("4x0e+4x1o+4x1e+4x2e", 4), ("1x0e", 1),
          ("1x1o", 1), ("128x0e+128x1o", 8), ("96x0e+96x1o+96x2e", 3), ("2x4e+2x0e+2x8e", 1), ("130x0e+65x1o", 1), ("300x0e+20x0o", 20), ("16x0e+32x1o+16x2e", 16)]
# groups that a wave's registers do not hold, and many groups
LARGE = [("5000x0e+300x8e", 1), ("700x0e+512x3o", 1), ("512x0e+512x1o", 256), ("96x0e+192x1o", 48)]
GRAPHS = [None, [0, 27], [0, 1, 1, 3, 40, 41], [2, 2, 9, 35], [0, 0]]


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("ir_mul", [False, True])
@pytest.mark.parametrize("irreps,groups", IRREPS)
def test_against_the_oracle(irreps, groups, ir_mul, prec):
    # without gates in one layout each (a normalisation takes seconds to compile where its code is not cached)
    for gated in (True, False) if (IRREPS.index((irreps, groups)) % 2 == 0) == ir_mul and prec == "f32" else (True,):
        n = handle(irreps, groups, layer.SILU, gated, prec, ir_mul)
        for i, ptr in enumerate(GRAPHS):
            N = 41 if ptr is not None else 37
            p = inputs(n, N, prec, seed=i)
            compare(run(n, p, ptr), irreps, groups, layer.SILU, gated, ir_mul, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("irreps,groups", LARGE)
def test_large_groups(irreps, groups, prec):
    n = handle(irreps, groups, layer.SILU, True, prec, groups == 256)
    for ptr in (None, [0, 5, 5, 11], [0, 12]):
        p = inputs(n, 12, prec, seed=3)
        compare(run(n, p, ptr), irreps, groups, layer.SILU, True, groups == 256, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("act", [layer.NONE, layer.GELU, layer.SIGMOID, layer.TANH])
def test_activations(act, prec):
    irreps = "12x0e+4x1o"
    n = handle(irreps, 2, act, True, prec, False)
    for ptr in (None, [0, 9, 20]):
        p = inputs(n, 20, prec, seed=act)
        compare(run(n, p, ptr), irreps, 2, act, True, False, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("N,ptr", [(1, None), (700, None), (5000, [0, 5000]), (3000, [0, 1, 2, 2900, 2990, 3000]), (2600, [100 + 5 * i for i in range(501)]),
                                   (1500, [0] * 700 + [1500]), (513, [0, 256, 512, 513])])
def test_lengths(N, ptr, prec):
    irreps = "16x0e+8x1o+8x2e"
    n = handle(irreps, 2, layer.SILU, True, prec, True)
    p = inputs(n, N, prec, seed=N)
    compare(run(n, p, ptr), irreps, 2, layer.SILU, True, True, p, prec, ptr)


@pytest.mark.parametrize("prec", ["f32", "f64"])
def test_many_samples_without_rows(prec):
    """In front of the rows, between them, inside a chunk and behind the last; and no rows at all."""
    irreps = "16x0e+8x1o+8x2e"
    n = handle(irreps, 2, layer.SILU, True, prec, True)
    p = inputs(n, 400, prec, seed=5)
    own = [3, 7, 300, 400]       # ends of the samples with rows; rows 0 .. 2 belong to none
    ptr = sum(([v] * m for v, m in zip(own, (30_000, 70, 40_000, 25_000))), [])
    got, few = run(n, p, ptr), run(n, p, own)
    for name in ("y", "gx", "gweight", "gbias"):
        assert torch.equal(torch.nan_to_num(got[name]), torch.nan_to_num(few[name])), name
    have = torch.tensor([e > s for s, e in zip(ptr, ptr[1:])], device="cuda")
    assert torch.equal(got["stats"][have], few["stats"])
    none = got["stats"][~have].view(-1, n.n_stat // 2, 2)
    r = torch.tensor(1 / np.sqrt(1e-5), dtype=none.dtype, device="cuda")
    assert (none[..., 0] == 0).all() and torch.allclose(none[..., 1], r, rtol=1e-6, atol=0)
    got = run(n, [p[0][:0], p[1], p[2], p[3][:0]], [0] * 50_001)
    assert torch.allclose(got["stats"].view(50_000, -1, 2)[..., 1], r, rtol=1e-6, atol=0) and (got["gweight"] == 0).all() and (got["gbias"] == 0).all()


@pytest.mark.parametrize("prec,shift", [("f32", 1000.0), ("f64", 1e6)])
def test_far_from_zero(prec, shift):
    """Scalars whose mean is far larger than their spread: the variance is not the difference of two large numbers."""
    irreps = "32x0e"
    n = handle(irreps, 2, layer.NONE, True, prec, False)
    for ptr in (None, [0, 400, 801]):
        p = inputs(n, 801, prec, seed=1, shift=shift, scale=1.0)
        compare(run(n, p, ptr), irreps, 2, layer.NONE, True, False, p, prec, ptr)


def test_one_large_value_among_small_ones():
    irreps = "32x0e+8x1o"
    n = handle(irreps, 1, layer.SILU, True, "f32", False)
    for row, col in ((0, 0), (77, 3), (299, 31)):
        p = inputs(n, 300, "f32", seed=2)
        p[0][row, col] = 1e4
        for ptr in (None, [0, 300]):
            compare(run(n, p, ptr), irreps, 1, layer.SILU, True, False, p, "f32", ptr)


def test_constant_rows():
    """Variance zero: the results are the biases' activations, the gradients stay finite."""
    irreps = "8x0e+4x1o"
    n = handle(irreps, 1, layer.SILU, True, "f32", False)
    for ptr in (None, [0, 6]):
        p = inputs(n, 6, "f32", seed=3)
        p[0][:] = 0.5
        p[0][:, 8:20] = 0.0
        got = run(n, p, ptr)
        compare(got, irreps, 1, layer.SILU, True, False, p, "f32", ptr)
        assert (got["y"][:, 8:] == 0).all()


def test_nan_and_infinity_stay_in_their_unit():
    """A bad number spoils its sample's group and no other."""
    irreps = "8x0e+8x1o"
    for ptr in (None, [0, 10, 20]):
        n = handle(irreps, 2, layer.SILU, True, "f32", False)
        p = inputs(n, 20, "f32", seed=4)
        ref = run(n, p, ptr)
        for bad in (float("nan"), float("inf"), float("-inf")):
            q = [a.copy() for a in p]
            q[0][3, 1] = bad       # first group of the scalars
            got = run(n, q, ptr)
            hit = torch.zeros(20, dtype=torch.bool)
            hit[[3] if ptr is None else list(range(10))] = True
            assert torch.equal(got["y"][~hit], ref["y"][~hit]) and torch.equal(got["gx"][~hit], ref["gx"][~hit])
            assert torch.equal(got["y"][:, 4:], ref["y"][:, 4:]) and torch.isnan(got["y"][hit][:, :4]).any()
            assert torch.equal(got["gweight"][4:], ref["gweight"][4:])


def test_statistics_may_be_left_out():
    from paper_2501_13986_amd import binding as b
    n = handle("8x0e+8x1o", 2, layer.SILU, True, "f32", False)
    p = inputs(n, 50, "f32")
    x, w, bias, _ = [torch.from_numpy(a).cuda() for a in p]
    for ptr in (None, [0, 20, 50]):
        y = torch.empty((50, n.dim_y), device="cuda")
        b.norm_forward(n, x, w, bias, y, ptr=None if ptr is None else torch.tensor(ptr, device="cuda"))
        assert torch.equal(y, run(n, p, ptr)["y"])


def test_ptr_out_of_range_stays_inside():
    """Indices outside [0, N] are taken for the nearest inside; samples whose end is before their start are empty."""
    n = handle("8x0e+8x1o", 2, layer.SILU, True, "f32", False)
    p = inputs(n, 30, "f32")
    a, c = run(n, p, [-5, 10, 99]), run(n, p, [0, 10, 30])
    for k in a:
        assert torch.equal(a[k], c[k]), k
    run(n, p, [0, 20, 10, 30, 5, 1 << 40])     # decreasing: unspecified, but within the arrays


def test_no_rows():
    n = handle("8x0e+8x1o", 2, layer.SILU, True, "f32", False)
    for ptr in (None, [0], [0, 0, 0]):
        got = run(n, inputs(n, 0, "f32"), ptr)
        assert (got["gweight"] == 0).all() and (got["gbias"] == 0).all()
        if ptr is not None and len(ptr) > 1:
            st = got["stats"].reshape(2, -1, 2)
            assert (st[..., 0] == 0).all() and torch.allclose(st[..., 1], torch.full_like(st[..., 1], 1e5 ** 0.5))


def test_differences():
    """Gradients of a random direction against differences of the forward pass itself."""
    from paper_2501_13986_amd import binding as b
    n = handle("8x0e+8x1o+4x2e", 2, layer.SILU, True, "f64", True)
    for ptr in (None, [0, 7, 7, 20]):
        p = inputs(n, 20, "f64", seed=5)
        got = run(n, p, ptr)
        rng = np.random.default_rng(1)
        d = [rng.normal(size=a.shape) for a in p[:3]]
        t = None if ptr is None else torch.tensor(ptr, device="cuda")
        y, gy = torch.empty((20, n.dim_y), dtype=torch.float64, device="cuda"), torch.from_numpy(p[3]).cuda()

        def loss(h):
            q = [torch.from_numpy(a + h * v).cuda() for a, v in zip(p[:3], d)]
            b.norm_forward(n, *q, y, ptr=t)
            return float((y * gy).sum())

        h = 1e-4
        num = (loss(h) - loss(-h)) / (2 * h)
        terms = [got[k] * torch.from_numpy(v).cuda() for k, v in zip(("gx", "gweight", "gbias"), d)]
        ana, size = sum(float(v.sum()) for v in terms), sum(float(v.abs().sum()) for v in terms)
        assert abs(num - ana) <= 1000 * h * h * size


def test_runs_are_bit_identical():
    n = handle("32x0e+32x1o", 4, layer.SILU, True, "f32", False)
    p = inputs(n, 4000, "f32")
    for ptr in (None, [0, 4000], [0, 5, 1200, 4000]):
        a, c = run(n, p, ptr), run(n, p, ptr)
        for k in a:
            assert torch.equal(a[k], c[k]) or torch.isnan(a[k]).any(), k


def test_captured_and_replayed_on_two_streams():
    from paper_2501_13986_amd import binding as b
    n = handle("32x0e+32x1o+32x2e", 4, layer.SILU, True, "f32", True)
    for ptr in (None, [0, 30, 31, 200]):
        p = inputs(n, 200, "f32")
        x, w, bias, gy = [torch.from_numpy(a).cuda() for a in p]
        t = None if ptr is None else torch.tensor(ptr, device="cuda")
        S = 200 if ptr is None else 3
        new = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
        o = dict(y=new(200, n.dim_y), stats=new(S, n.n_stat), gx=new(200, n.dim_x), gweight=new(n.n_w), gbias=new(n.n_b))

        def step():
            b.norm_forward(n, x, w, bias, o["y"], o["stats"], ptr=t)
            b.norm_backward(n, x, w, bias, gy, o["stats"], o["gx"], o["gweight"], o["gbias"], ptr=t)

        step()
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph):
            step()
        for seed in (21, 22, 23):
            q = inputs(n, 200, "f32", seed=seed)
            for dst, src in zip((x, w, bias, gy), q):
                dst.copy_(torch.from_numpy(src))
            for v in o.values():
                v.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            with torch.cuda.stream(side):      # an eager call on another stream at the same time, buffers of its own
                ref = run(n, q, ptr)
            torch.cuda.synchronize()
            for k in ref:
                assert torch.equal(ref[k], o[k]), k


def test_offsets_beyond_32_bits():
    """Rows behind the first 2^31 elements and 2^32 bytes."""
    from paper_2501_13986_amd import binding as b
    irreps, N = "128x0e+128x1o+128x2e+128x3o", 1_060_000
    n = handle(irreps, 1, layer.SILU, True, "f32", False)
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((N, n.dim_x), generator=g, device="cuda")
    w, bias = torch.rand(n.n_w, generator=g, device="cuda") + 0.5, torch.rand(n.n_b, generator=g, device="cuda")
    gy = torch.zeros((N, n.dim_y), device="cuda")
    at = [0, 883_011, 883_012, 1_048_576, N - 1]
    gy[at] = torch.randn((len(at), n.dim_y), generator=g, device="cuda")
    for ptr in (None, [0, 883_000, 883_020, 1_048_570, N]):
        t = None if ptr is None else torch.tensor(ptr, device="cuda")
        S = N if ptr is None else 4
        y, stats = torch.full((N, n.dim_y), float("nan"), device="cuda"), torch.empty((S, n.n_stat), device="cuda")
        gx, gw, gb = torch.full((N, n.dim_x), float("nan"), device="cuda"), torch.empty(n.n_w, device="cuda"), torch.empty(n.n_b, device="cuda")
        b.norm_forward(n, x, w, bias, y, stats, ptr=t)
        b.norm_backward(n, x, w, bias, gy, stats, gx, gw, gb, ptr=t)
        assert not torch.isnan(y[::4099]).any() and not torch.isnan(gx[::4099]).any() and not torch.isnan(y[-1]).any() and not torch.isnan(gx[-1]).any()
        if ptr is None:
            p = [v.cpu().numpy() for v in (x[at], w, bias, gy[at])]
            got = dict(y=y[at], stats=stats[at], gx=gx[at], gweight=gw, gbias=gb)
            compare(got, irreps, 1, layer.SILU, True, False, p, "f32", None)
        else:
            s, e = ptr[1], ptr[2]
            p = [v.cpu().numpy() for v in (x[s:e], w, bias, gy[s:e])]
            ref = layer.norm(irreps, 1, layer.SILU, True, 1e-5, False, *p[:3], [0, e - s], p[3])
            for k, v in (("y", y[s:e]), ("gx", gx[s:e]), ("stats", stats[1:2])):
                check(v.cpu().numpy().reshape(ref[k][0].shape), ref[k], norm_tolerance(ref[k], "f32", 1), k)
        del y, gx
