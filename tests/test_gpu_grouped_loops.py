"""The inner loops of the products by kind of row at sizes that reach them: many lines a workgroup, full tiles, long chunks, rows and matrices beyond 32 bits, several launches.

References are in fp64 on the GPU, group by group; bounds count the roundings that follow one another, so that a row left out is seen."""
import numpy as np
import pytest

from paper_2501_13986_amd import binding as b
from tests import _grouped_paths as paths
from tests._products import EPS

torch = pytest.importorskip("torch")
DT = {"f32": torch.float32, "f64": torch.float64}
PRECS = ["f32", "f64"]
gpu = pytest.mark.gpu


def inputs(rows, K, n, sizes, prec, comps=1, perm=False, front=0, seed=0, ld=None):
    """On the GPU.  ld: x, gx, gout and out are columns of one array whose rows are so wide."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=DT[prec])  # noqa: E731
    p = dict(W=draw(len(sizes), K, n), ptr=front + torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), device="cuda"), perm=torch.randperm(rows, generator=g, device="cuda") if perm else None,
             comps=comps, prec=prec, sizes=list(sizes))
    assert int(p["ptr"][-1]) <= rows
    if ld is None:
        p.update(x=draw(rows, comps * K), gout=draw(rows, comps * n), out=torch.full((rows, comps * n), float("nan"), device="cuda", dtype=DT[prec]),
                 gx=torch.full((rows, comps * K), float("nan"), device="cuda", dtype=DT[prec]))
    else:
        big, at = torch.empty(rows * ld, device="cuda", dtype=DT[prec]), 0
        for name, w in (("x", K), ("gout", n), ("out", n), ("gx", K)):
            p[name] = big.as_strided((rows, comps * w), (ld, 1), at)
            p[name].copy_(draw(rows, comps * w)) if name in ("x", "gout") else p[name].fill_(float("nan"))
            at += comps * w
        assert at <= ld
    return p


def run(p):
    print(*(f"{k}={tuple(v.shape)}/{v.stride(0)}" for k, v in p.items() if k in ("x", "W", "gout")), f"comps={p['comps']} perm={p['perm'] is not None} {p['prec']}", flush=True)
    gW = torch.full_like(p["W"], float("nan"))
    b.grouped_forward(p["x"], p["W"], p["out"], p["ptr"], perm=p["perm"], comps=p["comps"])
    b.grouped_backward(p["x"], p["W"], p["gout"], p["gx"], gW, p["ptr"], perm=p["perm"], comps=p["comps"])
    torch.cuda.synchronize()
    return gW


def compare(p, gW, names=("out", "gx", "gW")):
    rows, (groups, K, n), comps, prec = p["x"].shape[0], p["W"].shape, p["comps"], p["prec"]
    cuts = p["ptr"].tolist()
    perm = torch.arange(rows, device="cuda") if p["perm"] is None else p["perm"]
    for g in range(groups):
        at = perm[cuts[g]:cuts[g + 1]]
        x, t, W = p["x"][at].double().reshape(-1, K), p["gout"][at].double().reshape(-1, n), p["W"][g].double()
        ref = {"out": (x @ W, x.abs() @ W.abs()), "gx": (t @ W.T, t.abs() @ W.abs().T), "gW": (x.T @ t, x.abs().T @ t.abs())}
        got = {"out": p["out"][at].double().reshape(-1, n), "gx": p["gx"][at].double().reshape(-1, K), "gW": gW[g].double()}
        tol = paths.tolerances(ref, rows, K, n, comps, max(1, at.shape[0]), prec)
        for name in names:
            off = (got[name] - ref[name][0]).abs()
            ok = off <= tol[name]      # not where it is NaN
            assert bool(ok.all()), f"group {g} {name}: {int((~ok).sum())} of {ok.numel()} off, first at {(~ok).nonzero()[0].tolist()}, {off[~ok][0].item():.3g} for {tol[name][~ok][0].item():.3g}"
    rest = torch.cat([perm[:cuts[0]], perm[cuts[-1]:]])
    assert bool(torch.isnan(p["out"][rest]).all()) and bool(torch.isnan(p["gx"][rest]).all())


def filled(head, rows, piece):
    """Sizes: those of `head`, then pieces of at most `piece` that fill the rows but nine."""
    left = rows - 9 - sum(head)
    return list(head) + [piece] * (left // piece) + [left % piece]


# remainders of 64 and of 16 lines, of a workgroup's lines, empty and tiny groups
HEAD = [64 * 5 + 1, 64 * 7 + 16, 64 * 3 + 17, 0, 1, 1024 * 2, 1024 * 5 + 1, 1024 + 63, 15, 17, 64 * 2 + 48, 0, 64 * 9 + 49]
# rows, K, n, comps: workgroups of 1024 lines forward, for each number of parts of the matrix that a wave may keep
STREAM = [(1_050_003, 8, 12, 1), (150_003, 9, 13, 7), (530_003, 40, 65, 1), (1_050_003, 70, 3, 1), (1_050_003, 128, 5, 1)]
# full tiles: more than 128 terms, forward or backward
FULL = [(70_001, 130, 40), (70_001, 132, 40), (70_001, 41, 131), (70_001, 40, 132)]
# chunks of more than 512 lines; groups that end just behind 512 lines of a chunk
CHUNKS = [(30_011, 301, 299, 1), (30_011, 300, 300, 1), (6011, 300, 301, 7), (140_011, 64, 2176, 1)]
CHUNK_HEAD = {1: [513, 511 + 544, 480 + 545, 479 + 512, 1024, 1, 100, 0, 2900, 31, 513], 7: [74, 54 + 78, 50 + 73, 55, 128, 1, 10, 0, 560, 4, 74]}


@pytest.mark.parametrize("prec", PRECS)
def test_sizes_take_the_loops_they_are_meant_for(prec):
    for rows, K, n, comps in STREAM:
        for perm in (False, True):
            how, lines = paths.lines_of_products(rows, K, n, comps, perm, comps * K, comps * n, K * n, prec)
            assert how == "stream" and lines >= (1024 if n < 64 else 512)
    for rows, K, n in FULL:
        back = K <= 128
        assert paths.lines_of_products(rows, n if back else K, K if back else n, 1, True, n if back else K, K if back else n, K * n, prec) == ("rows", paths.TILE[prec])
    for rows, K, n, comps in CHUNKS:
        assert paths.positions_of_a_chunk(rows, K, n, comps, prec) * comps > 512


def test_the_workspace_is_that_of_the_rules():
    for rows in (1, 100, 3000, 20_000, 30_011, 160_710):
        for K, n, comps in ((64, 2176, 1), (128, 128, 7), (301, 299, 1), (20, 33, 1), (300, 301, 7), (3, 1, 2)):
            for prec in PRECS:
                assert b.lib().cgtp_grouped_workspace_bytes(rows, K, n, comps, 5, b.CGTP_F64 if prec == "f64" else b.CGTP_F32) == paths.workspace(rows, K, n, comps, prec)


@gpu
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,K,n,comps", STREAM)
def test_many_lines_a_workgroup(rows, K, n, comps, prec):
    for perm in (False, True):
        p = inputs(rows, K, n, filled(HEAD, rows, 40_000), prec, comps=comps, perm=perm, front=4, seed=K)
        compare(p, run(p))


@gpu
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,K,n", FULL)
def test_full_tiles(rows, K, n, prec):
    for perm in (False, True):
        p = inputs(rows, K, n, filled(HEAD, rows, 9000), prec, perm=perm, front=5, seed=n)
        compare(p, run(p))


# ---- the matrices' gradients: a row that is left out, or counted twice, is seen

SUMS = [(rows, K, n, comps, filled(CHUNK_HEAD[comps], rows, 4000 // comps)) for rows, K, n, comps in CHUNKS] + [
    (9000, 20, 33, 1, [10, 4000, 0, 256, 4700]), (3000, 36, 20, 3, [2999]), (20_003, 64, 64, 1, [1, 5000, 63, 4999, 65, 5000, 4800]), (5000, 130, 200, 1, [4999])]


def outer_products(rows, K, n, comps, size, prec):
    """Sizes of a position's share of gW, and the bound for a group of so many positions."""
    rng = np.random.default_rng(rows)
    most = min(size, 500)
    x, t = rng.normal(size=(most, comps, K)), rng.normal(size=(most, comps, n))
    magnitude = np.abs(x).reshape(-1, K).T @ np.abs(t).reshape(-1, n) * (size / most)
    return np.abs(x[0].T @ t[0]), paths.tolerances({k: (None, magnitude) for k in ("out", "gx", "gW")}, rows, K, n, comps, size, prec)["gW"]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,K,n,comps,sizes", SUMS)
def test_a_row_left_out_is_seen(rows, K, n, comps, sizes, prec):
    one, tol = outer_products(rows, K, n, comps, max(sizes), prec)
    assert (one > 2 * tol).mean() > 0.5


@gpu
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,K,n,comps,sizes", SUMS)
def test_every_row_counts_once(rows, K, n, comps, sizes, prec):
    for perm in (False, True):
        front = min(7, rows - sum(sizes))      # chunks are of positions: groups begin anywhere in them
        for f in {0, front}:
            p = inputs(rows, K, n, sizes, prec, comps=comps, perm=perm, front=f, seed=rows + f)
            compare(p, run(p))


# ---- rows and matrices beyond 32 bits

@gpu
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("K,n,comps", [(40, 24, 1), (20, 33, 3), (150, 131, 1)])
def test_arrays_beyond_32_bits_without_a_permutation(K, n, comps, prec):
    """Each workgroup's rows are within 2^31 bytes, all of them are not."""
    rows, ld = 6000, 1_000_000 // paths.SIZE[prec] + 1
    assert rows * ld * paths.SIZE[prec] > 2 ** 32 and paths.near(paths.reached(rows, comps, False), ld, prec)
    p = inputs(rows, K, n, [5, 2000, 0, 3300, 650], prec, comps=comps, front=20, seed=K, ld=ld)
    compare(p, run(p))


@gpu
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("K,n,comps", [(40, 24, 1), (21, 33, 3), (150, 130, 1)])
def test_rows_far_apart(K, n, comps, perm, prec):
    """Rows of one workgroup are 2^31 bytes apart and more."""
    rows, ld = 1100, (1 << 23) // paths.SIZE[prec]
    assert not paths.near(paths.reached(rows, comps, perm), ld, prec)
    p = inputs(rows, K, n, [500, 0, 70, 519], prec, comps=comps, perm=perm, front=3, seed=K, ld=ld)
    compare(p, run(p))


@gpu
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,n", [(3, 16_500), (70, 16_501)])
def test_matrices_beyond_32_bits(rows, n, prec):
    K = (1 << 17) // paths.SIZE[prec]
    assert not paths.near(K, n, prec)
    p = inputs(rows, K, n, [rows - 1, 1], prec, perm=True, seed=rows)
    p["W"].mul_(0.01)
    compare(p, run(p))


@gpu
@pytest.mark.parametrize("prec", PRECS)
def test_more_groups_than_a_launch_has_workgroups(prec):
    groups, rows = (1 << 23) + 70, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=DT[prec])  # noqa: E731
    x, W, gout = draw(rows, 3), draw(groups, 3, 2), draw(rows, 2)
    kinds = torch.cat([torch.randint(0, groups, (rows - 60,), generator=g, device="cuda"), torch.arange(groups - 60, groups, device="cuda")]).sort().values
    ptr = torch.searchsorted(kinds, torch.arange(groups + 1, device="cuda"))
    out, gx, gW = torch.full_like(gout, float("nan")), torch.full_like(x, float("nan")), torch.full_like(W, float("nan"))
    b.grouped_forward(x, W, out, ptr)
    b.grouped_backward(x, W, gout, gx, gW, ptr)
    Wk, xd, td = W[kinds].double(), x.double(), gout.double()
    for got, want in ((out, (xd[:, :, None] * Wk).sum(1)), (gx, (td[:, None, :] * Wk).sum(2)),
                      (gW, torch.zeros(groups, 3, 2, dtype=torch.float64, device="cuda").index_add_(0, kinds, xd[:, :, None] * td[:, None, :]))):
        assert bool(((got.double() - want).abs() <= EPS[prec] * 200 * 3 * 40).all())
        assert bool(((got == 0) == (want == 0)).all())
