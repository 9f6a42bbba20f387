"""The gated feed-forward block against the fp64 oracle."""
import numpy as np
import pytest

from oracle import layer
from tests._layer import EPS, check, gated_tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DT = {"f32": torch.float32, "f64": torch.float64}
NAMES = ("gx", "gWg", "gWu", "gbg", "gbu")


def inputs(rows, k, n, prec, bias, seed=0, spread=0.0):
    rng = np.random.default_rng(seed)
    draw = lambda *s: rng.normal(size=s) * np.exp(spread * rng.normal(size=s))  # noqa: E731
    p = [draw(rows, k), draw(k, n) / np.sqrt(k), draw(k, n) / np.sqrt(k)] + ([draw(n), draw(n)] if bias else [None, None]) + [draw(rows, n)]
    return [None if a is None else a.astype(np.float32 if prec == "f32" else np.float64) for a in p]


def dev(a, wide=0, fill=7.0):
    """On the GPU; wide: as the first columns of rows that are so much wider."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if not wide:
        return t
    w = torch.full((t.shape[0], t.shape[1] + wide), fill, dtype=t.dtype, device="cuda")
    w[:, :t.shape[1]] = t
    return w[:, :t.shape[1]]


def outputs(rows, k, n, prec, bias, wide=0):
    new = lambda *s: torch.full(s, float("nan"), dtype=DT[prec], device="cuda")  # noqa: E731
    return (new(rows, n + wide)[:, :n], new(rows, k + wide)[:, :k], new(k, n), new(k, n)) + ((new(n), new(n)) if bias else (None, None))


def run(p, prec, act, bias, wide=0):
    from paper_2501_13986_amd import binding as b
    x, Wg, Wu, bg, bu, gout = p
    rows, (k, n) = x.shape[0], Wg.shape
    t = [dev(x, wide), dev(Wg), dev(Wu), dev(bg), dev(bu)]
    o = outputs(rows, k, n, prec, bias, wide)
    b.gated_forward(t[0], t[1], t[2], o[0], bg=t[3], bu=t[4], act=act)
    b.gated_backward(t[0], t[1], t[2], dev(gout, wide), o[1], o[2], o[3], bg=t[3], bu=t[4], gbg=o[4], gbu=o[5], act=act)
    torch.cuda.synchronize()
    return o


def compare(o, p, prec, act, what):
    x, Wg, Wu, bg, bu, gout = p
    ref = layer.gated(x, Wg, Wu, bg, bu, act, gout)
    for name, got in zip(("out",) + NAMES, o):
        if got is not None:
            check(got.cpu().numpy(), ref[name], gated_tolerance(ref[name], prec, Wg.shape[0], Wg.shape[1], x.shape[0]), f"{what} {name}")


# one of everything, around the tiles' edges, and the widths of this library's plans
SIZES = [(1, 1, 1), (2, 64, 544), (1, 8, 24), (5, 3, 2), (31, 16, 33), (33, 8, 17), (64, 64, 64), (65, 37, 301), (243, 8, 160), (300, 64, 96),
         (129, 130, 65), (64, 256, 33), (1000, 16, 130), (31, 128, 127), (257, 5, 64), (128, 200, 7), (97, 129, 40), (1030, 64, 31), (8300, 136, 40), (300, 96, 100), (2100, 70, 129), (700, 33, 270), (2000, 8, 70), (1500, 5, 33), (90, 16, 48), (5000, 12, 20), (33, 10, 100), (1300, 20, 64)]


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_against_the_oracle(rows, k, n, prec):
    bias = (rows + n) % 2 == 0
    p = inputs(rows, k, n, prec, bias)
    compare(run(p, prec, layer.SILU, bias), p, prec, layer.SILU, f"{rows}x{k}x{n}")


@pytest.mark.parametrize("rows,k,n,prec", [(40_000, 16, 70, "f32"), (20_000, 14, 70, "f64"), (33_000, 100, 97, "f32"), (16_500, 128, 65, "f64")])
def test_uneven_shares_are_split(rows, k, n, prec):
    """A few workgroups more than compute units: the columns of W are split for gx."""
    p = inputs(rows, k, n, prec, True, seed=rows)
    compare(run(p, prec, layer.SILU, True), p, prec, layer.SILU, (rows, k, n))


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("act", [layer.NONE, layer.GELU, layer.SIGMOID, layer.TANH])
@pytest.mark.parametrize("k", [7, 14, 20, 40, 80, 110, 140])
def test_activations(k, act, prec):
    p = inputs(70, k, 50, prec, True, seed=act)
    compare(run(p, prec, act, True), p, prec, act, f"act {act}")


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,k,n,wide", [(40, 24, 36, 4), (33, 7, 19, 1), (100, 64, 64, 3), (1, 64, 64, 64), (150, 150, 70, 5), (20, 100, 30, 2)])
def test_columns_of_wider_rows(rows, k, n, wide, prec):
    """What lies between the rows is not touched."""
    p = inputs(rows, k, n, prec, False, seed=2)
    o = run(p, prec, layer.SILU, False, wide)
    compare(o, p, prec, layer.SILU, "strided")
    for t, w in ((o[0], n), (o[1], k)):
        whole = t.as_strided((rows, w + wide), (w + wide, 1))
        assert torch.isnan(whole[:, w:]).all()


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("rows,k,n,wide", [(70, 7, 19, 3), (65, 30, 33, 2), (130, 61, 66, 1), (20, 101, 30, 5), (140, 131, 35, 3), (64, 10, 9, 7), (64, 15, 18, 1)])
def test_what_lies_between_rows_is_not_used(rows, k, n, wide, prec):
    """NaN behind every row, whose widths end inside a load of four numbers."""
    p = inputs(rows, k, n, prec, True, seed=k)
    from paper_2501_13986_amd import binding as b
    x, gout = dev(p[0], wide, float("nan")), dev(p[5], wide, float("nan"))
    t = [dev(a) for a in p[1:5]]
    o = outputs(rows, k, n, prec, True, wide)
    b.gated_forward(x, *t[:2], o[0], bg=t[2], bu=t[3])
    b.gated_backward(x, *t[:2], gout, o[1], o[2], o[3], bg=t[2], bu=t[3], gbg=o[4], gbu=o[5])
    compare(o, p, prec, layer.SILU, (rows, k, n, wide))
    for out, w in ((o[0], n), (o[1], k)):
        assert torch.isnan(out.as_strided((rows - 1, wide), (w + wide, 1), w)).all()


@pytest.mark.parametrize("prec", ["f32", "f64"])
def test_numbers_far_apart(prec):
    """Factors over many powers of two: each product keeps the precision of its type."""
    p = inputs(50, 48, 40, prec, True, seed=9, spread=4.0)
    compare(run(p, prec, layer.NONE, True), p, prec, layer.NONE, "spread")


@pytest.mark.parametrize("k", [8, 16, 64, 200])
@pytest.mark.parametrize("power", [100, 115, 126, 140])
def test_smallest_numbers(k, power):
    """A part of a factor below 2^-126 counts as zero: two parts of it at most, so a factor is off by 2^-125 at most."""
    p = inputs(64, k, 64, "f32", True, seed=power)
    p[0] = (p[0].astype(np.float64) * 2.0 ** -power).astype(np.float32)
    p[2][:], p[3][:], p[4][:] = 0, 0, 1        # out = x Wg
    out = run(p, "f32", layer.NONE, True)[0].cpu().numpy()
    ref = layer.gated(*p[:5], layer.NONE, p[5])["out"]
    check(out, ref, gated_tolerance(ref, "f32", k, 64, 64) + 2.0 ** -125 * np.abs(p[1].astype(np.float64)).sum(0), "out")


def test_infinities_and_nan_stay_in_their_rows():
    p = inputs(70, 20, 40, "f32", False, seed=4)
    ref = run(p, "f32", layer.SILU, False)
    x = p[0].copy()
    x[3, 5], x[40, 0], x[69, 19] = np.inf, np.nan, -np.inf
    o = run([x] + p[1:], "f32", layer.SILU, False)
    clean = [r for r in range(70) if r not in (3, 40, 69)]
    assert torch.equal(o[0][clean], ref[0][clean]) and torch.equal(o[1][clean], ref[1][clean])
    for r in (3, 40, 69):
        assert not torch.isfinite(o[0][r]).any()


def test_saturated_activations():
    from paper_2501_13986_amd import binding as b
    x = torch.tensor([[1000.0], [-1000.0], [200.0], [-90.0], [0.0]], device="cuda")
    one = torch.ones((1, 1), device="cuda")
    out = torch.empty((5, 1), device="cuda")
    b.gated_forward(x, one, one, out, act=b.ACT_SILU)
    assert torch.allclose(out.double(), x.double() ** 2 * torch.sigmoid(x.double()), rtol=1e-6, atol=1e-30)
    b.gated_forward(x, one, one, out, act=b.ACT_SIGMOID)
    assert torch.allclose(out.double(), x.double() * torch.sigmoid(x.double()), rtol=1e-6, atol=1e-30)


def test_no_rows():
    p = inputs(0, 8, 16, "f32", True)
    o = run(p, "f32", layer.SILU, True)
    for t in o[2:]:
        assert (t == 0).all()


@pytest.mark.parametrize("prec", ["f32", "f64"])
def test_differences(prec):
    """Gradients of a random direction against differences of the forward pass itself."""
    from paper_2501_13986_amd import binding as b
    p = inputs(64, 24, 40, "f64", True, seed=6)
    o = run([a.astype(np.float32) if prec == "f32" else a for a in p], prec, layer.SILU, True)
    rng = np.random.default_rng(1)
    d = [rng.normal(size=a.shape) for a in p[:5]]
    out = torch.empty((64, 40), dtype=torch.float64, device="cuda")

    def loss(h):
        t = [dev(a + h * v) for a, v in zip(p[:5], d)]
        b.gated_forward(t[0], t[1], t[2], out, bg=t[3], bu=t[4])
        return float((out * dev(p[5])).sum())

    h = 1e-4
    num = (loss(h) - loss(-h)) / (2 * h)
    ana = sum(float((g.double() * dev(v)).sum()) for g, v in zip(o[1:], d))
    size = sum(float((g.double() * dev(v)).abs().sum()) for g, v in zip(o[1:], d))
    # the differences' own error is h^2 times third derivatives of the terms, fewer than 100 of them per number
    assert abs(num - ana) <= (100 * h * h + 400 * EPS[prec]) * size


def test_runs_are_bit_identical():
    p = inputs(5000, 64, 160, "f32", True, seed=8)
    a, c = run(p, "f32", layer.SILU, True), run(p, "f32", layer.SILU, True)
    for s, t in zip(a, c):
        assert torch.equal(s, t)


def test_another_stream_and_two_at_once():
    from paper_2501_13986_amd import binding as b
    ps = [inputs(3000, 64, 96, "f32", False, seed=s) for s in (1, 2)]
    ref = [run(p, "f32", layer.SILU, False) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    ts = [[dev(a) for a in p] for p in ps]
    os_ = [outputs(3000, 64, 96, "f32", False) for _ in ps]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, t, o in zip(streams, ts, os_):
            with torch.cuda.stream(s):
                b.gated_forward(t[0], t[1], t[2], o[0])
                b.gated_backward(t[0], t[1], t[2], t[5], o[1], o[2], o[3])
    torch.cuda.synchronize()
    for r, o in zip(ref, os_):
        for s, t in zip(r[:4], o[:4]):
            assert torch.equal(s, t)


def test_captured_and_replayed():
    from paper_2501_13986_amd import binding as b
    p = inputs(700, 32, 96, "f32", True, seed=3)
    t = [dev(a) for a in p]
    o = outputs(700, 32, 96, "f32", True)

    def step():
        b.gated_forward(t[0], t[1], t[2], o[0], bg=t[3], bu=t[4])
        b.gated_backward(t[0], t[1], t[2], t[5], o[1], o[2], o[3], bg=t[3], bu=t[4], gbg=o[4], gbu=o[5])

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (11, 12, 13):
        q = inputs(700, 32, 96, "f32", True, seed=seed)
        for dst, src in zip(t, q):
            dst.copy_(dev(src))
        for v in o:
            v.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for s, v in zip(run(q, "f32", layer.SILU, True), o):
            assert torch.equal(s, v)


def test_offsets_beyond_32_bits():
    """More than 2^31 elements between the first and the last row, and more than 4 GiB of results."""
    from paper_2501_13986_amd import binding as b
    rows, k, n = 1_050_000, 8, 2080
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((rows, k), generator=g, device="cuda")
    W = [torch.randn((k, n), generator=g, device="cuda") for _ in range(2)]
    out = torch.full((rows, n), float("nan"), device="cuda")
    b.gated_forward(x, *W, out)
    gout = torch.zeros((rows, n), device="cuda")
    at = [0, 1, 524_287, 1_032_444, 1_032_445, rows - 2, rows - 1]
    gout[at] = torch.randn((len(at), n), generator=g, device="cuda")
    gx, gW = torch.full_like(x, float("nan")), [torch.empty_like(w) for w in W]
    b.gated_backward(x, *W, gout, gx, *gW)
    ref = layer.gated(x[at].cpu().numpy(), *[w.cpu().numpy() for w in W], None, None, layer.SILU, gout[at].cpu().numpy())
    for name, got in (("out", out[at]), ("gx", gx[at]), ("gWg", gW[0]), ("gWu", gW[1])):
        check(got.cpu().numpy(), ref[name], gated_tolerance(ref[name], "f32", k, n, len(at)), name)
    assert not torch.isnan(out[::4099]).any() and not torch.isnan(out[-1]).any() and not torch.isnan(gx).any()


def sparse_gout(rows, n, at, dtype, gen):
    gout = torch.zeros((rows, n), dtype=dtype, device="cuda")
    gout[at] = torch.randn((len(at), n), generator=gen, dtype=dtype, device="cuda")
    return gout


def test_more_rows_than_one_launch_has_threads_for():
    """2^30 rows and some: 64 to a workgroup of 256 threads."""
    from paper_2501_13986_amd import binding as b
    rows = (1 << 30) + 70
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, 1), generator=g, dtype=torch.float64, device="cuda")
    W = [torch.randn((1, 1), generator=g, dtype=torch.float64, device="cuda") for _ in range(2)]
    at = [0, 63, (1 << 28) - 1, 1 << 28, (1 << 29) + 5, (1 << 30) - 1, 1 << 30, rows - 1]
    gout = sparse_gout(rows, 1, at, torch.float64, g)
    gx, gW = torch.full_like(x, float("nan")), [torch.empty_like(w) for w in W]
    b.gated_backward(x, *W, gout, gx, *gW)
    ref = layer.gated(x[at].cpu().numpy(), *[w.cpu().numpy() for w in W], None, None, layer.SILU, gout[at].cpu().numpy())
    for name, got in (("gx", gx[at]), ("gWg", gW[0]), ("gWu", gW[1])):
        check(got.cpu().numpy(), ref[name], gated_tolerance(ref[name], "f64", 1, 1, len(at)), name)
    assert not torch.isnan(gx).any()
    del gout, gx
    out = torch.full_like(x, float("nan"))
    b.gated_forward(x, *W, out)
    check(out[at].cpu().numpy(), ref["out"], gated_tolerance(ref["out"], "f64", 1, 1, len(at)), "out")
    assert not torch.isnan(out).any()


def test_more_weights_than_one_launch_has_threads_for():
    """2 * 2048 * 2^20 sums: a row of 2047 numbers, 2^20 columns."""
    from paper_2501_13986_amd import binding as b
    k, n = 2047, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((1, k), generator=g, device="cuda")
    W = [torch.randn((k, n), generator=g, device="cuda") for _ in range(2)]
    at = [0, 1, 255, 256, 524_287, n - 2, n - 1]     # columns of gout that are not zero
    gout = torch.zeros((1, n), device="cuda")
    gout[:, at] = torch.randn((1, len(at)), generator=g, device="cuda")
    gx, gW = torch.full_like(x, float("nan")), [torch.full_like(w, float("nan")) for w in W]
    b.gated_backward(x, *W, gout, gx, *gW)
    ref = layer.gated(x.cpu().numpy(), *[w[:, at].cpu().numpy() for w in W], None, None, layer.SILU, gout[:, at].cpu().numpy())
    for name, got in (("gx", gx), ("gWg", gW[0][:, at]), ("gWu", gW[1][:, at])):
        check(got.cpu().numpy(), ref[name], gated_tolerance(ref[name], "f32", k, len(at), 1), name)
    for t in gW:
        assert not torch.isnan(t[::97]).any() and not torch.isnan(t[-1]).any() and (t[:, 2] == 0).all()
