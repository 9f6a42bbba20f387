"""Products by kind of row and orthogonalised updates: sizes, inputs, one pass of each, and what a pass cannot do without.

  grouped   rows of one kind (species of the nodes, pair types of the edges) share a matrix: out = x W[kind] (+ b[kind]), a segment of
            several components in the layout IR_MUL component by component; rows are sorted by kind, or stay where they are and are
            reached through a permutation.  Operations: fwd (inference), bwd (the gradients alone), step (both)
  orth      the update of a batch of weights is orthogonalised: X = G / (|G| + eps), then some steps X <- a X + (b A + c A A) X with
            A = X X^T, which take all singular values close to one

The plain forms are elementary torch operations; `own` makes the calls of `paper_2501_13986_amd.binding`.
"""
from __future__ import annotations

from math import log, sqrt

import torch

own = False

EPS = 1e-7
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def listed():
    return [
        # the three atoms of a water molecule in a model for 89 elements: one evaluation, latency alone
        {"name": "grouped fwd, 3 atoms", "kind": "grouped", "op": "fwd", "dtype": "f32", "rows": 3, "pad": 0, "groups": 89, "d_in": 128, "d_out": 128, "comps": 1, "bias": False, "perm": True, "wide": 0},
        # one molecule of 27 atoms, four elements: training
        {"name": "grouped step, small molecule", "kind": "grouped", "op": "step", "dtype": "f32", "rows": 27, "pad": 0, "groups": 4, "d_in": 64, "d_out": 64, "comps": 1, "bias": True, "perm": True, "wide": 0},
        # the vectors of a protein-sized graph, 89 elements: inference
        {"name": "grouped fwd, 20000 nodes", "kind": "grouped", "op": "fwd", "dtype": "f32", "rows": 20000, "pad": 0, "groups": 89, "d_in": 128, "d_out": 128, "comps": 3, "bias": False, "perm": True, "wide": 0},
        # the l = 3 segment of the same, columns of wider rows, ten elements: training, padded to a fixed number of nodes
        {"name": "grouped step, 20000 nodes", "kind": "grouped", "op": "step", "dtype": "f32", "rows": 20000, "pad": 480, "groups": 10, "d_in": 128, "d_out": 128, "comps": 7, "bias": False, "perm": True, "wide": 1152},
        # the edges of the same, sorted by pair type, to all weights of the benchmark's convolution: inference, and the largest case
        {"name": "grouped fwd, 160710 edges", "kind": "grouped", "op": "fwd", "dtype": "f32", "rows": 160710, "pad": 0, "groups": 25, "d_in": 64, "d_out": 2176, "comps": 1, "bias": False, "perm": False, "wide": 0},
        {"name": "grouped bwd, 160710 edges", "kind": "grouped", "op": "bwd", "dtype": "f32", "rows": 160710, "pad": 0, "groups": 25, "d_in": 64, "d_out": 2176, "comps": 1, "bias": False, "perm": False, "wide": 0},
        # double precision, odd widths, biases
        {"name": "grouped step f64, 2503 nodes", "kind": "grouped", "op": "step", "dtype": "f64", "rows": 2503, "pad": 0, "groups": 17, "d_in": 96, "d_out": 301, "comps": 1, "bias": True, "perm": True, "wide": 0},
        # a hidden layer of a radial network: latency alone
        {"name": "orth, 64 x 64", "kind": "orth", "dtype": "f32", "batch": 1, "m": 64, "n": 64, "steps": 5, "absent": 0},
        # both matrices of the gated block that puts out all weights of the benchmark's convolution
        {"name": "orth, 2 of 64 x 2176", "kind": "orth", "dtype": "f32", "batch": 2, "m": 64, "n": 2176, "steps": 5, "absent": 0},
        # one matrix for each of 89 elements, of which some were not in the batch
        {"name": "orth, 89 of 128 x 128", "kind": "orth", "dtype": "f32", "batch": 89, "m": 128, "n": 128, "steps": 5, "absent": 7},
        # a dense map between whole rows of the benchmark's convolution
        {"name": "orth, 1152 x 2048", "kind": "orth", "dtype": "f32", "batch": 1, "m": 1152, "n": 2048, "steps": 5, "absent": 0},
        # double precision, more rows than columns, odd
        {"name": "orth f64, 17 of 301 x 96", "kind": "orth", "dtype": "f64", "batch": 17, "m": 301, "n": 96, "steps": 5, "absent": 2},
    ]


def _spread(rng, low, high):
    """A whole number spread over its logarithm."""
    return min(high, max(low, int(round(2 ** rng.uniform(log(low, 2), log(high, 2))))))


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        c = {"kind": rng.choice(["grouped", "grouped", "orth"]), "dtype": rng.choice(["f32", "f32", "f64"])}
        if c["kind"] == "grouped":
            c["op"] = rng.choice(["fwd", "bwd", "step"])
            c["rows"], c["groups"] = _spread(rng, 1, 160710), _spread(rng, 1, 400)
            c["d_in"], c["d_out"] = _spread(rng, 1, 512), _spread(rng, 1, 2176)
            c["comps"] = rng.choice([1, 1, 1, 3, 5, 7])
            c["bias"] = c["comps"] == 1 and rng.random() < 0.5
            c["perm"] = rng.random() < 0.6
            c["pad"] = rng.choice([0, 0, rng.randint(1, 500)])
            c["wide"] = rng.randint(1, 1152) if rng.random() < 0.3 else 0
        else:
            c["batch"], c["m"], c["n"] = _spread(rng, 1, 400), _spread(rng, 1, 2176), _spread(rng, 1, 2176)
            c["steps"] = rng.choice([3, 5, 5, 6])
            c["absent"] = rng.choice([0, rng.randint(0, c["batch"] // 4)])
        if _seconds(c) <= most:
            return c


def _seconds(case):
    """A measure of a case's cost (only to keep the drawn ones below the largest listed one)."""
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / (8e13 if case["dtype"] == "f32" else 4e13))


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float64 if case["dtype"] == "f64" else torch.float32
    draw_ = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=dt)  # noqa: E731
    if case["kind"] == "orth":
        # gradients: small, rows and columns of unlike sizes, none where no row of a kind was seen
        B, m, n = case["batch"], case["m"], case["n"]
        G = draw_(B, m, n) * torch.exp(0.5 * draw_(B, m, 1)) * torch.exp(0.5 * draw_(B, 1, n)) * 1e-3
        if case["absent"]:
            G[torch.randperm(B, generator=g, device="cuda")[:case["absent"]]] = 0
        return {"G": G}
    N, E, K, n, C, all_ = case["rows"], case["groups"], case["d_in"], case["d_out"], case["comps"], case["rows"] + case["pad"]
    # a few kinds are frequent, many are rare, some are absent
    often = 1 / torch.arange(1, E + 1, device="cuda", dtype=torch.float64)
    kinds = torch.multinomial(often[torch.randperm(E, generator=g, device="cuda")], N, replacement=True, generator=g)
    if not case["perm"]:
        kinds = kinds.sort().values
    s = {"kinds": kinds, "ptr": torch.cat([kinds.new_zeros(1), torch.bincount(kinds, minlength=E).cumsum(0)]), "perm": None}
    if case["perm"]:        # rows behind the last one belong to no kind
        s["perm"] = torch.cat([torch.sort(kinds, stable=True).indices, torch.arange(N, all_, device="cuda")])
    s["x"] = draw_(all_, C * K + case["wide"])[:, :C * K]
    s["W"] = draw_(E, K, n).mul_(1 / sqrt(K))
    s["b"] = draw_(E, n).mul_(0.1) if case["bias"] else None
    if case["op"] != "fwd":
        s["gout"] = draw_(all_, C * n)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "orth":
        s["coefficients"] = [COEFFICIENTS] * case["steps"]
        if own:
            from paper_2501_13986_amd import binding as b
            s["lib"], s["out"] = b, torch.empty_like(s["G"])
        return s
    if not own:
        s["cuts"] = s["ptr"].tolist()
        return s
    from paper_2501_13986_amd import binding as b
    all_, C = case["rows"] + case["pad"], case["comps"]
    s["lib"] = b
    s["out"] = s["x"].new_zeros((all_, C * case["d_out"]))
    s["gx"] = s["x"].new_zeros((all_, C * case["d_in"]))
    s["gW"] = torch.empty_like(s["W"])
    s["gb"] = torch.empty_like(s["b"]) if case["bias"] else None
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    case, back = s["case"], ()
    if not own:
        return (_orth if case["kind"] == "orth" else _grouped)(s)
    b = s["lib"]
    if case["kind"] == "orth":
        return b.orthogonalise(s["G"], s["out"], coefficients=s["coefficients"], eps=EPS)
    if case["op"] != "bwd":
        back += (b.grouped_forward(s["x"], s["W"], s["out"], s["ptr"], b=s["b"], perm=s["perm"], comps=case["comps"]),)
    if case["op"] != "fwd":
        g = b.grouped_backward(s["x"], s["W"], s["gout"], s["gx"], s["gW"], s["ptr"], gb=s["gb"], perm=s["perm"], comps=case["comps"])
        back += tuple(t for t in g if t is not None)
    return back


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _grouped(s):
    case, cuts, W, perm = s["case"], s["cuts"], s["W"], s["perm"]
    K, n, C, N = case["d_in"], case["d_out"], case["comps"], case["rows"]
    fwd, bwd = case["op"] != "bwd", case["op"] != "fwd"
    x = s["x"]
    out = x.new_zeros((x.shape[0], C * n)) if fwd else None
    if bwd:
        gx, gW = x.new_zeros((x.shape[0], C * K)), torch.zeros_like(W)
        gb = torch.zeros_like(s["b"]) if case["bias"] else None
    for e in range(case["groups"]):
        lo, hi = cuts[e], cuts[e + 1]
        if lo == hi:
            continue
        at = slice(lo, hi) if perm is None else perm[lo:hi]
        rows = x[at].reshape(-1, K)
        if fwd:
            v = rows @ W[e]
            if case["bias"]:
                v = v + s["b"][e]
            out[at] = v.reshape(-1, C * n)
        if bwd:
            t = s["gout"][at].reshape(-1, n)
            gx[at] = (t @ W[e].T).reshape(-1, C * K)
            gW[e] = rows.T @ t
            if case["bias"]:
                gb[e] = t.double().sum(0).to(t.dtype)
    return ((out,) if fwd else ()) + ((gx, gW) + ((gb,) if case["bias"] else ()) if bwd else ())


def _orth(s):
    G = s["G"]
    wide = G.shape[1] <= G.shape[2]
    X = G.double() / (G.double().square().sum((1, 2), keepdim=True).sqrt() + EPS)
    X = (X if wide else X.transpose(1, 2)).to(G.dtype).contiguous()
    for a, b, c in s["coefficients"]:
        A = X @ X.transpose(1, 2).contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X if wide else X.transpose(1, 2).contiguous()


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    el = 8 if case["dtype"] == "f64" else 4
    if case["kind"] == "orth":
        B, s, l = case["batch"], min(case["m"], case["n"]), max(case["m"], case["n"])
        # A and A A are symmetric: half of their products
        return {"bytes": 2 * B * s * l * el, "flops": B * case["steps"] * (3 * s * s * l + s * s * s)}
    N, E, K, n, C = case["rows"], case["groups"], case["d_in"], case["d_out"], case["comps"]
    fwd, bwd = case["op"] != "bwd", case["op"] != "fwd"
    used, bias = min(E, N) * K * n, n if case["bias"] else 0
    moved = (N * C * (K + n) + used + min(E, N) * bias if fwd else 0) + (N * C * (2 * K + n) + used + E * (K * n + bias) if bwd else 0)
    index = 8 * (E + 1 + (N if case["perm"] else 0))
    return {"bytes": moved * el + index, "flops": 2 * N * C * K * n * ((1 if fwd else 0) + (2 if bwd else 0))}


# ---- the same from the definitions, 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "orth":
        return _exact_orth(case, s["G"].double())
    K, n, C = case["d_in"], case["d_out"], case["comps"]
    E, all_ = case["groups"], case["rows"] + case["pad"]
    fwd, bwd = case["op"] != "bwd", case["op"] != "fwd"
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, gx, gW, gb = new(all_, C, n) if fwd else None, new(all_, C, K) if bwd else None, new(E, K, n), new(E, n)
    for kind in s["kinds"].unique().tolist():
        members = (s["kinds"] == kind).nonzero()[:, 0]
        for part in members.split(16384):
            x = s["x"][part].double().reshape(-1, C, K).requires_grad_(bwd)
            W = s["W"][kind].double().requires_grad_(bwd)
            b = (s["b"][kind].double() if case["bias"] else new(n)).requires_grad_(bwd)
            v = torch.tensordot(x, W, 1) + b
            if fwd:
                out[part] = v.detach()
            if bwd:
                t = s["gout"][part].double().reshape(-1, C, n)
                d = torch.autograd.grad((v * t).sum(), (x, W, b))
                gx[part] = d[0]
                gW[kind] += d[1]
                gb[kind] += d[2]
    back = (out.reshape(all_, C * n),) if fwd else ()
    if bwd:
        back += (gx.reshape(all_, C * K), gW) + ((gb,) if case["bias"] else ())
    return back


def _exact_orth(case, G):
    """The steps from the other side of the matrix or with another association: X (a + b M + c M M) with M = X^T X has the same value."""
    a, b, c = COEFFICIENTS
    X = G / (torch.linalg.vector_norm(G, dim=(1, 2), keepdim=True) + EPS)
    few = X.shape[2] < X.shape[1]
    for _ in range(case["steps"]):
        T = X.transpose(1, 2).contiguous()
        if few:
            Y = X @ (T @ X)
            X = a * X + b * Y + c * (Y @ (T @ X))
        else:
            A = X @ T
            Y = A @ X
            X = a * X + b * Y + c * (A @ Y)
    return X
