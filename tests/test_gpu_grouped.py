"""The products by kind of row against the fp64 oracle."""
import numpy as np
import pytest

from oracle import products
from tests._products import check, grouped_tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DT = {"f32": torch.float32, "f64": torch.float64}
NP = {"f32": np.float32, "f64": np.float64}
PRECS = ["f32", "f64"]


def dev(a, wide=0, fill=float("nan")):
    """On the GPU; wide: as the first columns of rows that are so much wider."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if not wide:
        return t
    w = torch.full((t.shape[0], t.shape[1] + wide), fill, dtype=t.dtype, device="cuda")
    w[:, :t.shape[1]] = t
    return w[:, :t.shape[1]]


def inputs(rows, K, n, sizes, prec, comps=1, bias=False, perm=False, seed=0, spread=0.0, front=0):
    """sizes: rows of each group, behind `front` rows of none; what is left of the rows belongs to none."""
    rng = np.random.default_rng(seed)
    draw = lambda *s: (rng.normal(size=s) * np.exp(spread * rng.normal(size=s))).astype(NP[prec])  # noqa: E731
    ptr = front + np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    assert ptr[-1] <= rows
    return dict(x=draw(rows, comps * K), W=draw(len(sizes), K, n), b=draw(len(sizes), n) if bias else None, gout=draw(rows, comps * n), ptr=ptr,
                perm=rng.permutation(rows).astype(np.int64) if perm else None, comps=comps, prec=prec)


def run(p, wide=0):
    from paper_2501_13986_amd import binding as b
    new = lambda *s: torch.full(s, float("nan"), dtype=DT[p["prec"]], device="cuda")  # noqa: E731
    (rows, ck), (groups, K, n), comps = p["x"].shape, p["W"].shape, p["comps"]
    print(f"rows={rows} K={K} n={n} groups={groups} comps={comps} perm={p['perm'] is not None} bias={p['b'] is not None} wide={wide} {p['prec']}", flush=True)
    x, W, ptr, perm = dev(p["x"], wide), dev(p["W"]), dev(p["ptr"]), dev(p["perm"])
    out, gx = new(rows, comps * n + wide)[:, :comps * n], new(rows, ck + wide)[:, :ck]
    gW, gb = new(groups, K, n), new(groups, n) if p["b"] is not None else None
    b.grouped_forward(x, W, out, ptr, b=dev(p["b"]), perm=perm, comps=comps)
    b.grouped_backward(x, W, dev(p["gout"], wide), gx, gW, ptr, gb=gb, perm=perm, comps=comps)
    torch.cuda.synchronize()
    return dict(out=out, gx=gx, gW=gW, gb=gb)


def compare(o, p, what=""):
    ref = products.grouped(p["x"], p["W"], p["ptr"], p["perm"], p["b"], p["comps"], p["gout"])
    (_, K, n), rows = p["W"].shape, p["x"].shape[0]
    for name, terms in (("out", K), ("gx", n), ("gW", rows * p["comps"]), ("gb", rows)):
        if o[name] is not None:
            check(o[name].cpu().numpy(), ref[name], grouped_tolerance(ref[name], p["prec"], terms), f"{what} {name}")


# rows, K, n, sizes of the groups: one of everything, around the tiles' edges, empty groups at the ends and between
SIZES = [
    (1, 1, 1, [1]), (3, 128, 128, [0, 1, 0, 2, 0]), (5, 3, 2, [0, 0, 5]), (64, 64, 64, [64]), (65, 32, 33, [1, 63, 1]), (130, 33, 65, [129, 0, 1]), (128, 31, 127, [127, 1]),
    (300, 64, 96, [128, 128, 44]), (300, 5, 7, [299]), (257, 130, 40, [3, 200, 0, 0, 54]), (1030, 64, 31, [1030]), (700, 200, 150, [256, 256, 188]), (129, 128, 301, [64, 65]), (600, 96, 3, [255, 257, 88]),
    (2, 1, 300, [1, 1]), (1500, 2, 129, [513, 0, 900]), (90, 257, 1, [30, 30, 30])]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,K,n,sizes", SIZES)
def test_against_the_oracle(rows, K, n, sizes, prec):
    for perm in (False, True):
        p = inputs(rows, K, n, sizes, prec, bias=(rows + n) % 2 == 0, perm=perm, seed=rows)
        compare(run(p), p)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("comps", [2, 3, 7, 17])
@pytest.mark.parametrize("rows,K,n,sizes", [(1, 5, 6, [1]), (50, 32, 32, [10, 0, 37]), (130, 64, 20, [63, 65]), (40, 131, 66, [20, 20]), (600, 8, 12, [300, 290])])
def test_components(rows, K, n, sizes, comps, prec):
    p = inputs(rows, K, n, sizes, prec, comps=comps, perm=True, seed=comps)
    compare(run(p), p)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("K,n,wide,comps", [(24, 36, 4, 1), (7, 19, 1, 1), (64, 64, 3, 3), (150, 70, 5, 1), (3, 2, 2, 5), (128, 128, 1152, 1)])
def test_columns_of_wider_rows(K, n, wide, comps, prec):
    """NaN lies between the rows of x and gout; what lies between those of the results is not touched."""
    p = inputs(140, K, n, [70, 0, 60], prec, comps=comps, bias=comps == 1, perm=True, seed=K)
    o = run(p, wide)
    compare(o, p)
    for t, w in ((o["out"], comps * n), (o["gx"], comps * K)):
        assert torch.isnan(t.as_strided((139, wide), (w + wide, 1), w)).all()


@pytest.mark.parametrize("prec", PRECS)
def test_rows_of_no_group_stay(prec):
    """In front of the first group and behind the last; `check` wants NaN there."""
    for perm in (False, True):
        p = inputs(300, 40, 24, [100, 0, 90], prec, bias=True, perm=perm, front=60)
        compare(run(p), p)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("groups", [64, 65, 700, 5000])
def test_many_groups(groups, prec):
    rng = np.random.default_rng(groups)
    sizes = rng.integers(0, 4, groups) * (rng.random(groups) < 0.5)
    sizes[groups // 2] = 700
    p = inputs(int(sizes.sum()) + 5, 12, 9, sizes, prec, bias=True, perm=True, seed=groups)
    compare(run(p), p)


@pytest.mark.parametrize("prec", PRECS)
def test_groups_over_many_chunks(prec):
    p = inputs(9000, 20, 33, [10, 4000, 0, 256, 4700], prec, bias=True, perm=True, seed=5)
    compare(run(p), p)
    p = inputs(3000, 36, 20, [2999], prec, comps=3, seed=6)
    compare(run(p), p)


@pytest.mark.parametrize("prec", PRECS)
def test_all_groups_empty(prec):
    from paper_2501_13986_amd import binding as b
    for rows in (0, 40):
        p = inputs(rows, 6, 10, [0, 0, 0], prec, bias=True)
        o = run(p)
        assert torch.isnan(o["out"]).all() and torch.isnan(o["gx"]).all()
        assert not o["gW"].any() and not o["gb"].any()
    W = torch.zeros(0, 4, 4, dtype=DT[prec], device="cuda")
    b.grouped_forward(torch.zeros(3, 4, dtype=DT[prec], device="cuda"), W, torch.zeros(3, 4, dtype=DT[prec], device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"))


@pytest.mark.parametrize("prec", PRECS)
def test_positions_outside(prec):
    """Rows that perm does not name inside [0, rows) are left out, numbers of ptr outside are those of the ends."""
    p = inputs(200, 20, 24, [90, 70], prec, bias=True, perm=True)
    p["perm"][[3, 95, 140]] = [-1, 200, 1 << 40]
    p["ptr"] = np.array([-5, 90, 1 << 50], np.int64)
    compare(run(p), p)


@pytest.mark.parametrize("prec", PRECS)
def test_a_row_named_twice_holds_one_of_the_results(prec):
    p = inputs(150, 16, 20, [80, 70], prec, perm=True)
    p["perm"][100] = p["perm"][10]
    lost = sorted(set(range(150)) - set(p["perm"].tolist()))
    out = run(p)["out"].cpu().numpy()
    r, x, W = p["perm"][10], p["x"].astype(np.float64), p["W"].astype(np.float64)
    tol = 1e-5 if prec == "f32" else 1e-13
    assert min(np.abs(out[r] - x[r] @ W[g]).max() for g in (0, 1)) < tol * 100
    assert np.isnan(out[lost]).all() and not np.isnan(np.delete(out, lost, 0)).any()


@pytest.mark.parametrize("prec", PRECS)
def test_numbers_far_apart(prec):
    p = inputs(100, 48, 40, [30, 70], prec, bias=True, seed=9, spread=4.0)
    compare(run(p), p)


def test_infinities_and_nan_stay_in_their_rows_and_groups():
    p = inputs(150, 40, 36, [50, 60, 40], "f32", bias=True, perm=True, seed=3)
    ref = run(p)
    q = dict(p, x=p["x"].copy(), gout=p["gout"].copy())
    bad = [int(p["perm"][7]), int(p["perm"][100])]      # of groups 0 and 1
    q["x"][bad[0], 5], q["x"][bad[1], 39], q["gout"][bad[0], 1] = np.inf, np.nan, -np.inf
    o = run(q)
    clean = [r for r in range(150) if r not in bad]
    assert torch.equal(o["out"][clean], ref["out"][clean]) and torch.equal(o["gx"][clean], ref["gx"][clean])
    assert not torch.isfinite(o["out"][bad]).any() and not torch.isfinite(o["gx"][bad[0]]).any()
    assert torch.equal(o["gW"][2], ref["gW"][2]) and torch.equal(o["gb"][1:], ref["gb"][1:])
    assert not torch.isfinite(o["gW"][0, 5]).any() and not torch.isfinite(o["gW"][1, 39]).any() and not torch.isfinite(o["gb"][0, 1])
    assert torch.equal(o["gW"][1, :39], ref["gW"][1, :39])


@pytest.mark.parametrize("prec", PRECS)
def test_gradients_by_differences(prec):
    """The product is linear in each argument: a difference over a whole step is the gradient, up to roundings of the outputs."""
    from paper_2501_13986_amd import binding as b
    p = inputs(70, 12, 16, [30, 0, 38], prec, comps=1, bias=True, perm=True, seed=8)
    o = run(p)
    f = lambda **k: np.nansum(products.grouped(**{**{n: p[n] for n in ("x", "W", "ptr", "perm", "b", "comps")}, **k})["out"][0] * p["gout"])  # noqa: E731
    rng = np.random.default_rng(1)
    for name, at in (("gx", "x"), ("gW", "W"), ("gb", "b")):
        d = rng.normal(size=p[at].shape)
        want = f(**{at: p[at] + 0.5 * d}) - f(**{at: p[at] - 0.5 * d})
        got = np.nansum(o[name].cpu().numpy().astype(np.float64) * d)
        size = np.nansum(np.abs(o[name].cpu().numpy() * d))
        assert abs(got - want) <= (2.0 ** -24 if prec == "f32" else 2.0 ** -53) * (6 * 70 + 16) * 16 * size


def test_runs_repeat_bit_for_bit():
    p = inputs(5000, 70, 45, [100, 3000, 1200, 700], "f32", bias=True, perm=True, seed=2)
    a, b_ = run(p), run(p)
    assert all(torch.equal(a[k], b_[k]) for k in a)


@pytest.mark.parametrize("prec", PRECS)
def test_captured_and_replayed(prec):
    """New numbers and other groups in the same tensors; eager calls between the replays."""
    from paper_2501_13986_amd import binding as b
    p = inputs(2000, 24, 40, [500, 0, 1400], prec, bias=True, perm=True, seed=4)
    x, W, bias, gout, ptr, perm = (dev(p[k]) for k in ("x", "W", "b", "gout", "ptr", "perm"))
    new = lambda t: torch.full_like(t, float("nan"))  # noqa: E731
    o = dict(out=new(gout), gx=new(x), gW=new(W), gb=new(bias))

    def call(o):
        b.grouped_forward(x, W, o["out"], ptr, b=bias, perm=perm)
        b.grouped_backward(x, W, gout, o["gx"], o["gW"], ptr, gb=o["gb"], perm=perm)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(o)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):      # two graphs with workspaces of their own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(o)
        graphs.append(g)
    for i, sizes in enumerate([[500, 0, 1400], [3, 1990, 0], [0, 0, 2000], [700, 600, 650]]):
        q = inputs(2000, 24, 40, sizes, prec, bias=True, perm=True, seed=20 + i)
        for k, t in (("x", x), ("W", W), ("b", bias), ("gout", gout), ("ptr", ptr), ("perm", perm)):
            t.copy_(torch.from_numpy(q[k]))
        for t in o.values():
            t.fill_(float("nan"))
        graphs[i % 2].replay()
        other = {k: new(t) for k, t in o.items()}
        call(other)
        torch.cuda.synchronize()
        compare(o, q, f"replay {i}")
        assert all(torch.equal(torch.nan_to_num(o[k]), torch.nan_to_num(other[k])) for k in o)


def test_another_stream():
    from paper_2501_13986_amd import binding as b
    p = inputs(3000, 64, 64, [1000, 2000], "f32", perm=True)
    x, W, ptr, perm = (dev(p[k]) for k in ("x", "W", "ptr", "perm"))
    ref, outs, streams = torch.empty(3000, 64, device="cuda"), [torch.empty(3000, 64, device="cuda") for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    b.grouped_forward(x, W, ref, ptr, perm=perm)
    torch.cuda.synchronize()
    gW = [torch.empty_like(W) for _ in range(2)]
    for s, o, w in zip(streams, outs, gW):
        with torch.cuda.stream(s):
            b.grouped_forward(x, W, o, ptr, perm=perm)
            b.grouped_backward(x, W, o, torch.empty_like(x), w, ptr, perm=perm)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], ref) and torch.equal(outs[1], ref) and torch.equal(gW[0], gW[1])


def test_gradients_of_rows_beyond_32_bits():
    """Rows of x and gx lie up to 2^33 bytes apart, several chunks of a group."""
    from paper_2501_13986_amd import binding as b
    rows, ld = 1100, 1 << 21
    big = torch.empty(rows * ld, dtype=torch.float32, device="cuda")
    x, gx = big.as_strided((rows, 60), (ld, 1)), big.as_strided((rows, 60), (ld, 1), 1 << 20)
    p = inputs(rows, 20, 33, [500, 590], "f32", comps=3, perm=True, seed=1)
    x.copy_(torch.from_numpy(p["x"]))
    gx.fill_(float("nan"))
    gW = torch.empty(2, 20, 33, device="cuda")
    b.grouped_backward(x, dev(p["W"]), dev(p["gout"]), gx, gW, dev(p["ptr"]), perm=dev(p["perm"]), comps=3)
    torch.cuda.synchronize()
    compare(dict(out=None, gx=gx, gW=gW, gb=None), p, "far")


def test_rows_beyond_32_bits():
    """Rows of x and out lie up to 2^33 bytes apart."""
    from paper_2501_13986_amd import binding as b
    rows, ld = 1100, 1 << 21
    big = torch.empty(rows * ld, dtype=torch.float32, device="cuda")      # 9 GB, both x and out
    x, out = big.as_strided((rows, 40), (ld, 1)), big.as_strided((rows, 24), (ld, 1), 1 << 20)
    p = inputs(rows, 40, 24, [500, 590], "f32", perm=True, seed=1)
    x.copy_(torch.from_numpy(p["x"]))
    out.fill_(float("nan"))
    b.grouped_forward(x, dev(p["W"]), out, dev(p["ptr"]), perm=dev(p["perm"]))
    torch.cuda.synchronize()
    ref = products.grouped(p["x"], p["W"], p["ptr"], p["perm"])
    check(out.cpu().numpy(), ref["out"], grouped_tolerance(ref["out"], "f32", 40), "out")
