"""The layer operators around the convolution: sizes, inputs, one pass of each, and what a pass cannot do without.

  gated   the gated feed-forward block out = act(x Wg + bg) * (x Wu + bu): from the edges' scalars it forms the weights that the
          convolution reads (d_out = n_w of the plan), and its gradients start from those that the convolution returns
  norm    group normalisation of irreps rows with the activation and the gates behind the convolution: scalars are centred, scaled
          and put through the activation, the other segments are scaled by their root mean square and multiplied by the sigmoid of
          their gate; statistics per node, or over all nodes of a graph

Operations: fwd (inference), bwd (the gradients alone), step (both).  The plain forms are elementary torch operations; `own` makes
the calls of `paper_2501_13986_amd.binding`.
"""
from __future__ import annotations

from functools import lru_cache
from math import log, pi, sqrt

import torch

own = False

# irreps of the rows that are normalised: what the convolutions of this repository's benchmark and tests put out
IRREPS = {
    "mace": "128x0e+128x1o+128x2e+128x3o",
    "mul96": "96x0e+96x1o+96x2e",
    "mul32": "32x0e+32x1o+32x2e+32x3o",
    "nequip": "32x0e+32x1o+32x2e",
    "uneven": "16x0e+32x1o+16x2e",
    "diffdock": "48x0e+10x1o+10x1e+48x0o",
    "tiny": "4x0e+4x1o+4x1e+4x2e",
    "scalars": "128x0e",
    "odd": "7x0e+5x1o+3x2e+9x0e",
}
EPS = 1e-5


def listed():
    return [
        # the two edges of a dimer: one evaluation of its weights, latency alone
        {"name": "gated fwd, 2 edges", "kind": "gated", "op": "fwd", "dtype": "f32", "rows": 2, "d_in": 64, "d_out": 544, "act": "silu", "bias": False, "wide": 0},
        # one molecule of 27 atoms: energy and forces from eight radial functions
        {"name": "gated step, small molecule", "kind": "gated", "op": "step", "dtype": "f32", "rows": 243, "d_in": 8, "d_out": 544, "act": "silu", "bias": False, "wide": 0},
        # the edges of a protein-sized graph, all weights of the benchmark's convolution: inference
        {"name": "gated fwd, 160710 edges", "kind": "gated", "op": "fwd", "dtype": "f32", "rows": 160710, "d_in": 64, "d_out": 2176, "act": "silu", "bias": False, "wide": 0},
        # the same in training: the largest case
        {"name": "gated bwd, 160710 edges", "kind": "gated", "op": "bwd", "dtype": "f32", "rows": 160710, "d_in": 64, "d_out": 2176, "act": "silu", "bias": False, "wide": 0},
        # double precision, as reference comparisons run it
        {"name": "gated step f64, 30011 edges", "kind": "gated", "op": "step", "dtype": "f64", "rows": 30011, "d_in": 64, "d_out": 544, "act": "silu", "bias": True, "wide": 0},
        # the scalars of node rows (a slice of wider rows) to per-node weights: odd widths, biases, the other activation
        {"name": "gated step, 20011 nodes", "kind": "gated", "op": "step", "dtype": "f32", "rows": 20011, "d_in": 128, "d_out": 301, "act": "gelu", "bias": True, "wide": 1152},
        # one molecule: statistics over its 27 atoms
        {"name": "norm step, small molecule", "kind": "norm", "op": "step", "dtype": "f32", "rows": 27, "graphs": 1, "pad": 0, "irreps": "mul32", "layout": "mul_ir", "groups": 4, "act": "silu", "gated": True},
        # every node by itself: inference and training on the output of the benchmark's convolution
        {"name": "norm fwd, 20000 nodes", "kind": "norm", "op": "fwd", "dtype": "f32", "rows": 20000, "graphs": 0, "pad": 0, "irreps": "mace", "layout": "ir_mul", "groups": 1, "act": "silu", "gated": True},
        {"name": "norm step, 20000 nodes", "kind": "norm", "op": "step", "dtype": "f32", "rows": 20000, "graphs": 0, "pad": 0, "irreps": "mace", "layout": "mul_ir", "groups": 1, "act": "silu", "gated": True},
        # a training batch of molecules, padded to a fixed number of nodes
        {"name": "norm step, 500 molecules", "kind": "norm", "op": "step", "dtype": "f32", "rows": 12000, "graphs": 500, "pad": 313, "irreps": "mul32", "layout": "ir_mul", "groups": 4, "act": "silu", "gated": True},
        # one protein-sized graph as a whole
        {"name": "norm step, one graph of 20000", "kind": "norm", "op": "step", "dtype": "f32", "rows": 20000, "graphs": 1, "pad": 0, "irreps": "mace", "layout": "ir_mul", "groups": 8, "act": "silu", "gated": True},
        # double precision, odd multiplicities
        {"name": "norm step f64, 2503 nodes", "kind": "norm", "op": "step", "dtype": "f64", "rows": 2503, "graphs": 3, "pad": 0, "irreps": "odd", "layout": "mul_ir", "groups": 1, "act": "gelu", "gated": True},
    ]


def _spread(rng, low, high):
    """A whole number spread over its logarithm."""
    return min(high, max(low, int(round(2 ** rng.uniform(log(low, 2), log(high, 2))))))


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        c = {"kind": rng.choice(["gated", "norm"]), "op": rng.choice(["fwd", "bwd", "step"]), "dtype": rng.choice(["f32", "f32", "f64"]),
             "act": rng.choice(["silu", "silu", "gelu", "none"])}
        if c["kind"] == "gated":
            c["rows"], c["d_in"], c["d_out"] = _spread(rng, 1, 160710), _spread(rng, 4, 256), _spread(rng, 16, 2176)
            c["bias"] = rng.random() < 0.5
            c["wide"] = c["d_in"] + rng.randint(1, 1024) if rng.random() < 0.3 else 0
        else:
            c["rows"] = _spread(rng, 1, 30000)
            c["irreps"] = rng.choice(["mace", "mace", "mul96", "mul32", "nequip", "uneven", "diffdock", "tiny", "scalars", "odd"])
            c["layout"], c["gated"] = rng.choice(["mul_ir", "ir_mul"]), rng.random() < 0.7
            c["groups"] = rng.choice({"mace": [1, 2, 4, 8, 16, 32], "mul96": [1, 3, 8], "mul32": [1, 4, 8, 32], "nequip": [1, 2, 8], "uneven": [1, 2, 16],
                                      "diffdock": [1, 2], "tiny": [1, 2, 4], "scalars": [1, 8, 32], "odd": [1]}[c["irreps"]])
            per_node = rng.random() < 0.4
            c["graphs"] = 0 if per_node else _spread(rng, 1, max(1, c["rows"] // 8))
            c["pad"] = 0 if per_node else rng.choice([0, 0, rng.randint(1, 300)])
        if _seconds(c) <= most:
            return c


def _seconds(case):
    """A measure of a case's cost (only to keep the drawn ones below the largest listed one)."""
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / (8e13 if case["dtype"] == "f32" else 4e13))


# ---- the rows' description ----------------------------------------------------------------------------------------------

def _segments(case):
    """(mul, 2l+1, whether invariant, first column) of every segment; behind them the gates, scalars, one segment for each of the
    segments that are not invariant."""
    out, at = [], 0
    for t in IRREPS[case["irreps"]].split("+"):
        mul, ir = t.split("x")
        n = 2 * int(ir[:-1]) + 1
        out.append((int(mul), n, ir == "0e", at))
        at += int(mul) * n
    gates, dim_y = [], at
    for s in out:
        if case["gated"] and not s[2]:
            gates.append((s[0], 1, True, at))
            at += s[0]
    return out + gates, dim_y, at


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float64 if case["dtype"] == "f64" else torch.float32
    draw_ = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=dt)  # noqa: E731
    s, N = {}, case["rows"]
    if case["kind"] == "gated":
        K, n = case["d_in"], case["d_out"]
        if K == 8:      # radial functions sin(k pi r) / r of the edges' lengths, within the cutoff r = 1
            r = torch.rand((N, 1), generator=g, device="cuda", dtype=torch.float64) ** (1 / 3) * 0.9 + 0.1
            s["x"] = (sqrt(2.0) * torch.sin(r * (pi * torch.arange(1, K + 1, device="cuda", dtype=torch.float64))) / r).to(dt)
        else:           # activations of a layer before, or the first columns of wider rows
            s["x"] = draw_(N, case["wide"])[:, :K] if case["wide"] else draw_(N, K)
        s["Wg"], s["Wu"] = draw_(K, n).mul_(1 / sqrt(K)), draw_(K, n).mul_(1 / sqrt(K))
        s["bg"], s["bu"] = (draw_(n).mul_(0.1), draw_(n).mul_(0.1)) if case["bias"] else (None, None)
        if case["op"] != "fwd":
            s["gout"] = draw_(N, n)
        return s
    segs, dim_y, dim_x = _segments(case)
    # sums over a neighbourhood: a few units wide, the scalars off centre
    s["x"] = draw_(N + case["pad"], dim_x).mul_(4.0)
    for mul, n, inv, at in segs:
        if inv:
            s["x"][:, at:at + mul] += 1.5
    s["weight"] = draw_(sum(t[0] for t in segs)).mul_(0.1).add_(1.0)
    s["bias"] = draw_(sum(t[0] for t in segs if t[2])).mul_(0.1)
    if case["op"] != "fwd":
        s["gy"] = draw_(N + case["pad"], dim_y)
    S = case["graphs"]
    s["ptr"] = None
    if S:               # uneven graphs, now and then one without nodes; the rows behind the last one belong to none
        cuts = torch.randint(0, N + 1, (S - 1,), generator=g, device="cuda", dtype=torch.int64).sort().values
        s["ptr"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), N)])
    return s


@lru_cache(None)
def _handle(irreps, groups, act, gated, dtype, layout):
    """A program makes its normalisation when the model is defined and keeps it."""
    from paper_2501_13986_amd import binding as b
    return b.Norm(IRREPS[irreps], groups=groups, act=act, gated=gated, eps=EPS, dtype=b.CGTP_F64 if dtype == "f64" else b.CGTP_F32,
                  device=0, flags=b.CGTP_IR_MUL if layout == "ir_mul" else b.CGTP_MUL_IR)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "bwd" and case["kind"] == "norm":      # what the forward pass left
        s["stats"] = _statistics(case, s["x"], s["ptr"])
    elif case["kind"] == "norm":
        s["stats"] = torch.zeros((case["graphs"] or case["rows"], len(_segments(case)[0]), case["groups"], 2), dtype=s["x"].dtype, device="cuda")
    if not own:
        return s
    from paper_2501_13986_amd import binding as b
    like, zeros = torch.empty_like, torch.zeros_like
    s["b"], s["act"] = b, {"silu": b.ACT_SILU, "gelu": b.ACT_GELU, "none": b.ACT_NONE}[case["act"]]
    if case["kind"] == "gated":
        s["out"] = torch.empty((case["rows"], case["d_out"]), dtype=s["x"].dtype, device="cuda")
        s["gx"] = torch.empty((case["rows"], case["d_in"]), dtype=s["x"].dtype, device="cuda")
        s["gWg"], s["gWu"] = like(s["Wg"]), like(s["Wu"])
        s["gbg"], s["gbu"] = (like(s["bg"]), like(s["bu"])) if case["bias"] else (None, None)
        return s
    s["norm"] = _handle(case["irreps"], case["groups"], s["act"], case["gated"], case["dtype"], case["layout"])
    dim_y = _segments(case)[1]
    s["y"] = torch.zeros((s["x"].shape[0], dim_y), dtype=s["x"].dtype, device="cuda")
    s["gx"], s["gweight"], s["gbias"] = zeros(s["x"]), like(s["weight"]), like(s["bias"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    op, back = case["op"], ()
    if not own:
        return (_gated if case["kind"] == "gated" else _norm)(s)
    b = s["b"]
    if case["kind"] == "gated":
        if op != "bwd":
            back += (b.gated_forward(s["x"], s["Wg"], s["Wu"], s["out"], bg=s["bg"], bu=s["bu"], act=s["act"]),)
        if op != "fwd":
            g = b.gated_backward(s["x"], s["Wg"], s["Wu"], s["gout"], s["gx"], s["gWg"], s["gWu"], bg=s["bg"], bu=s["bu"], gbg=s["gbg"], gbu=s["gbu"], act=s["act"])
            back += tuple(t for t in g if t is not None)
        return back
    if op != "bwd":
        back += tuple(b.norm_forward(s["norm"], s["x"], s["weight"], s["bias"], s["y"], s["stats"], ptr=s["ptr"]))
    if op != "fwd":
        back += tuple(b.norm_backward(s["norm"], s["x"], s["weight"], s["bias"], s["gy"], s["stats"], s["gx"], s["gweight"], s["gbias"], ptr=s["ptr"]))
    return back


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _act(t, kind):
    """The activation and its derivative."""
    if kind == "silu":
        q = 1 / (1 + torch.exp(-t))
        return t * q, q * (1 + t * (1 - q))
    if kind == "gelu":      # t Phi(t), Phi(t) = (1 + erf(t / sqrt 2)) / 2
        p = 0.5 * (1 + torch.erf(t * sqrt(0.5)))
        return t * p, p + t * torch.exp(-0.5 * t * t) * (1 / sqrt(2 * pi))
    return t, torch.ones_like(t)


def _gated(s):
    case, x, Wg, Wu, out = s["case"], s["x"], s["Wg"], s["Wu"], ()
    g, u = x @ Wg, x @ Wu
    if case["bias"]:
        g, u = g + s["bg"], u + s["bu"]
    a, d = _act(g, case["act"])
    if case["op"] != "bwd":
        out += (a * u,)
    if case["op"] != "fwd":
        dg, du = s["gout"] * u * d, s["gout"] * a
        out += (dg @ Wg.T + du @ Wu.T, x.T @ dg, x.T @ du)
        if case["bias"]:
            out += (dg.double().sum(0).to(x.dtype), du.double().sum(0).to(x.dtype))
    return out


def _rows(case, ptr):
    """The graph of every row that belongs to one, and the number of graphs; rows by themselves: None."""
    if ptr is None:
        return None, case["rows"]
    return torch.repeat_interleave(torch.arange(case["graphs"], device=ptr.device), ptr[1:] - ptr[:-1], output_size=case["rows"]), case["graphs"]


def _per_graph(v, graph, S):
    """Sums of rows over graphs, 64 bits."""
    if S == 1:
        return v.sum(0, keepdim=True)
    return v if graph is None else torch.zeros((S,) + v.shape[1:], dtype=v.dtype, device=v.device).index_add_(0, graph, v)


def _of_rows(v, graph):
    return v if graph is None else v[graph]


def _columns(case, t, seg):
    """A segment as [rows, groups, channels of a group, components]."""
    mul, n, _, at = seg
    v = t[:case["rows"], at:at + mul * n]
    v = v.reshape(-1, n, mul).transpose(1, 2) if case["layout"] == "ir_mul" else v.reshape(-1, mul, n)
    return v.reshape(-1, case["groups"], mul // case["groups"], n)


def _back(case, v):
    """The columns of a segment given as [rows, groups, channels, components]."""
    v = v.reshape(v.shape[0], -1, v.shape[3])
    return (v.transpose(1, 2) if case["layout"] == "ir_mul" else v).reshape(v.shape[0], -1)


def _statistics(case, x, ptr):
    """Mean (invariant segments, else 0) and 1 / sqrt(variance + eps) [samples, segments, groups, 2], summed in 64 bits."""
    graph, S = _rows(case, ptr)
    rows = torch.ones(case["rows"], 1, dtype=torch.float64, device=x.device)
    rows, out = _per_graph(rows, graph, S).clamp(min=1), []
    for seg in _segments(case)[0]:
        v = _columns(case, x, seg).double()
        count = rows * (v.shape[2] * v.shape[3])
        mean = _per_graph(v.sum((2, 3)), graph, S) / count if seg[2] else torch.zeros_like(count).expand(S, case["groups"])
        var = _per_graph((v - _of_rows(mean, graph)[:, :, None, None]).square().sum((2, 3)), graph, S) / count
        out.append(torch.stack([mean, 1 / torch.sqrt(var + EPS)], 2))
    return torch.stack(out, 1).to(x.dtype)


def _norm(s):
    case, x, N = s["case"], s["x"], s["case"]["rows"]
    segs, dim_y, dim_x = _segments(case)
    op, G, out = case["op"], case["groups"], ()
    graph, S = _rows(case, s["ptr"])
    stats = _statistics(case, x, s["ptr"]) if op != "bwd" else s["stats"]
    hat, lin, weights, w_at, b_at = [], [], [], 0, 0      # normalised values, the same with weight and bias
    for k, seg in enumerate(segs):
        mul, _, inv, _ = seg
        t = _of_rows(stats[:, k], graph)
        hat.append((_columns(case, x, seg) - t[:, :, 0, None, None]) * t[:, :, 1, None, None])
        weights.append(s["weight"][w_at:w_at + mul].reshape(1, G, -1, 1))
        v = hat[-1] * weights[-1]
        lin.append(v + s["bias"][b_at:b_at + mul].reshape(1, G, -1, 1) if inv else v)
        w_at, b_at = w_at + mul, b_at + (mul if inv else 0)
    gates = dim_x > dim_y
    real = [t for t in segs if t[3] < dim_y]
    y, gx, glin, ggate = x.new_zeros((x.shape[0], dim_y)), torch.zeros_like(x), [], []
    gate_at = 0
    for k, seg in enumerate(real):
        mul, n, inv, at = seg
        gy = _columns(case, s["gy"], seg) if op != "fwd" else None
        if inv:
            a, d = _act(lin[k], case["act"])
            glin.append(gy * d if op != "fwd" else None)
        elif gates:
            q = 1 / (1 + torch.exp(-lin[len(real) + gate_at]))
            gate_at += 1
            a = lin[k] * q
            if op != "fwd":
                glin.append(gy * q)
                ggate.append((gy * lin[k]).sum(3, keepdim=True) * q * (1 - q))
        else:
            a = lin[k]
            glin.append(gy)
        if op != "bwd":
            y[:N, at:at + mul * n] = _back(case, a)
    if op != "bwd":
        out += (y, stats)
    if op == "fwd":
        return out
    glin += ggate
    rows = _per_graph(torch.ones(N, 1, dtype=torch.float64, device=x.device), graph, S).clamp(min=1)
    gw, gb = [], []
    for k, seg in enumerate(segs):
        mul, n, inv, at = seg
        gw.append((glin[k] * hat[k]).double().sum((0, 3)).reshape(-1))
        if inv:
            gb.append(glin[k].double().sum((0, 3)).reshape(-1))
        h = glin[k] * weights[k]
        count = rows * (mul // G * n)
        along = _of_rows(_per_graph((h * hat[k]).double().sum((2, 3)), graph, S) / count, graph).to(x.dtype)[:, :, None, None]
        v = h - hat[k] * along
        if inv:
            v = v - _of_rows(_per_graph(h.double().sum((2, 3)), graph, S) / count, graph).to(x.dtype)[:, :, None, None]
        gx[:N, at:at + mul * n] = _back(case, v * _of_rows(stats[:, k], graph)[:, :, 1, None, None])
    return out + (gx, torch.cat(gw).to(x.dtype), torch.cat(gb).to(x.dtype) if gb else x.new_zeros(0))


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    el = 8 if case["dtype"] == "f64" else 4
    fwd, bwd = case["op"] != "bwd", case["op"] != "fwd"
    if case["kind"] == "gated":
        R, K, n = case["rows"], case["d_in"], case["d_out"]
        weights, rows_in, rows_out = 2 * n * (K + (1 if case["bias"] else 0)), R * K, R * n
        # the forward's two products; the backward forms them again, and two for each of gx and the weights' gradients
        moved = (weights + rows_in + rows_out if fwd else 0) + (2 * weights + 2 * rows_in + rows_out if bwd else 0)
        return {"bytes": moved * el, "flops": R * K * n * ((4 if fwd else 0) + (12 if bwd else 0))}
    segs, dim_y, dim_x = _segments(case)
    R, S = case["rows"], case["graphs"] or case["rows"]
    stats = S * len(segs) * case["groups"] * 2
    params = sum(t[0] for t in segs) + sum(t[0] for t in segs if t[2])
    moved = (R * (dim_x + dim_y) + params + stats if fwd else 0) + (R * (2 * dim_x + dim_y) + 2 * params + stats if bwd else 0)
    return {"bytes": moved * el, "flops": R * dim_x * ((8 if fwd else 0) + (20 if bwd else 0))}


# ---- the same from the definitions, 64 bits, gradients by differentiation ----------------------------------------------

def _act64(t, kind):
    if kind == "none":
        return t
    return t / (1 + (-t).exp()) if kind == "silu" else t * (1 - 0.5 * torch.special.erfc(t / sqrt(2.0)))


def exact(case, seed):
    s = _inputs(case, seed)
    return (_exact_gated if case["kind"] == "gated" else _exact_norm)(case, {k: None if v is None else v if k == "ptr" else v.double() for k, v in s.items()})


def _exact_gated(case, s):
    R, leaves = case["rows"], [s[k] for k in ("Wg", "Wu") + (("bg", "bu") if case["bias"] else ())]
    sums = [torch.zeros_like(t) for t in leaves]
    outs, gxs = [], []
    for at in range(0, R, 16384):
        x = s["x"][at:at + 16384].clone().requires_grad_(True)
        ps = [t.clone().requires_grad_(True) for t in leaves]
        both = torch.mm(x, torch.cat(ps[:2], 1))
        if case["bias"]:
            both = both + torch.cat(ps[2:])
        o = _act64(both[:, :case["d_out"]], case["act"]) * both[:, case["d_out"]:]
        if case["op"] != "bwd":
            outs.append(o.detach())
        if case["op"] != "fwd":
            gr = torch.autograd.grad((o * s["gout"][at:at + 16384]).sum(), [x] + ps)
            gxs.append(gr[0])
            for t, v in zip(sums, gr[1:]):
                t += v
    return ((torch.cat(outs),) if case["op"] != "bwd" else ()) + ((torch.cat(gxs),) + tuple(sums) if case["op"] != "fwd" else ())


def _exact_norm(case, s):
    segs, dim_y, dim_x = _segments(case)
    N, G, pad = case["rows"], case["groups"], case["pad"]
    x, w, bias = (s[k].clone().requires_grad_(True) for k in ("x", "weight", "bias"))
    ids = torch.arange(N, device=x.device) if s["ptr"] is None else torch.bucketize(torch.arange(N, device=x.device), s["ptr"][1:], right=True)
    S = case["graphs"] or N
    size = torch.bincount(ids, minlength=S).double()
    # for each column: its channel and its group, from the layout
    pieces, stats, nw, nb = [], [], 0, 0
    for mul, n, inv, at in segs:
        col = torch.arange(mul * n, device=x.device)
        channel = col % mul if case["layout"] == "ir_mul" else col // n
        member = torch.nn.functional.one_hot(channel // (mul // G), G).double()          # [columns, groups]
        v = x[:N, at:at + mul * n]
        total = (size * (mul // G * n)).clamp(min=1)[:, None]
        mean = torch.zeros((S, G), dtype=v.dtype, device=v.device)
        if inv:
            mean = mean.index_add(0, ids, v @ member) / total
        c = v - (mean @ member.T)[ids]
        var = torch.zeros((S, G), dtype=v.dtype, device=v.device).index_add(0, ids, (c * c) @ member) / total
        r = (var + EPS) ** -0.5
        stats.append(torch.stack([mean, r], 2))
        t = c * (r @ member.T)[ids] * w[nw:nw + mul][channel]
        if inv:
            t = t + bias[nb:nb + mul][channel]
        pieces.append((t, channel))
        nw, nb = nw + mul, nb + (mul if inv else 0)
    y = []
    gates = [t for (_, _, _, at), (t, _) in zip(segs, pieces) if at >= dim_y]
    for (_, _, inv, at), (t, channel) in zip(segs, pieces):
        if at >= dim_y:
            break
        if inv:
            t = _act64(t, case["act"])
        elif gates:
            t = t * torch.sigmoid(gates.pop(0))[:, channel]
        y.append(t)
    y = torch.cat(y, 1)
    out = ()
    if case["op"] != "bwd":
        whole = torch.zeros((N + pad, dim_y), dtype=y.dtype, device=y.device)
        whole[:N] = y.detach()
        out += (whole, torch.stack(stats, 1).detach())
    if case["op"] != "fwd":
        gr = torch.autograd.grad((y * s["gy"][:N]).sum(), (x, w, bias), allow_unused=True, materialize_grads=True)
        out += tuple(gr)
    return out
