"""One interaction layer as a model runs it: weights of the edges by the gated block, the convolution, the normalisation with its
gates, and all of it backwards, against the fp64 oracles."""
import numpy as np
import pytest

from oracle import conv as oconv, layer
from oracle.irreps import TPSpec
from paper_2501_13986_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

NODE, EDGE, OUT = "16x0e+16x1o", "1x0e+1x1o+1x2e", "16x0e+16x1o+16x2e"
GATES = "+16x0e+16x0e"      # the convolution puts the gates out behind the irreps


@pytest.mark.parametrize("prec,tol", [("f32", 1e-4), ("f64", 1e-10)])
@pytest.mark.parametrize("ir_mul", [False, True])
def test_layer_forward_and_backward(prec, tol, ir_mul):
    """tol: the bars of this library's convolution, the least precise link."""
    from paper_2501_13986_amd import binding as b
    from tests._util import ir_mul_index
    dt = np.float32 if prec == "f32" else np.float64
    flags, code = (b.CGTP_IR_MUL if ir_mul else b.CGTP_MUL_IR), (b.CGTP_F64 if prec == "f64" else b.CGTP_F32)
    plan = b.Plan(NODE, EDGE, OUT + GATES, dtype=code, device=0, flags=flags)
    norm = b.Norm(OUT, groups=2, dtype=code, device=0, flags=flags)
    assert norm.dim_x == plan.dim_z
    spec = TPSpec(NODE, EDGE, OUT + GATES)
    V = 90
    recv, send, unit = synth.periodic_graph(1, V, 12.0)
    row_ptr, col, perm, t_row_ptr, t_perm = oconv.csr_from_coo(recv, send, V)
    E = recv.shape[0]
    y = synth.sh_edge_attr(unit[perm], 2).astype(dt)
    draw = lambda s, *shape: synth.normal(s, shape).astype(dt)  # noqa: E731
    x, a = draw(1, V, spec.dim_x), draw(2, E, 8)
    Wg, Wu, bg, bu = draw(3, 8, spec.n_w) / 3, draw(4, 8, spec.n_w) / 3, draw(5, spec.n_w), draw(6, spec.n_w)
    w, bias, gy = 1 + draw(7, norm.n_w) / 4, draw(8, norm.n_b) / 4, draw(9, V, norm.dim_y)
    ptr = [0, 40, 90]

    # oracle, default layout
    W = layer.gated(a, Wg, Wu, bg, bu, layer.SILU)["out"][0]
    z = oconv.forward(spec, x, y, W, row_ptr, col)
    n0 = layer.norm(OUT, 2, layer.SILU, True, 1e-5, False, z, w, bias, ptr, gy)
    rx, ry, rW = oconv.backward(spec, x, y, W, n0["gx"][0], row_ptr, col)
    rg = layer.gated(a, Wg, Wu, bg, bu, layer.SILU, rW)

    ix = {k: ir_mul_index(TPSpec(NODE, EDGE, OUT).irx if k == "x" else TPSpec(NODE, EDGE, OUT).irz) for k in "xy"}
    dev = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    lay = lambda v, k: v[:, ix[k]] if ir_mul else v  # noqa: E731
    new = lambda *s: torch.empty(s, dtype=torch.float64 if prec == "f64" else torch.float32, device="cuda")  # noqa: E731
    da, dWg, dWu, dbg, dbu, dx, dy = (dev(v) for v in (a, Wg, Wu, bg, bu, lay(x, "x"), y))
    dw, dbias, dgy, dptr = dev(w), dev(bias), dev(lay(gy, "y")), dev(np.asarray(ptr, np.int64))
    graph = [dev(v) for v in (row_ptr, col, t_row_ptr, t_perm)]
    W_, z_, y_, st = new(E, spec.n_w), new(V, spec.dim_z), new(V, norm.dim_y), new(2, norm.n_stat)
    gz, gx, gye, gW = new(V, spec.dim_z), new(V, spec.dim_x), new(E, spec.dim_y), new(E, spec.n_w)
    ga, gWg, gWu, gbg, gbu, gw, gb = new(E, 8), new(8, spec.n_w), new(8, spec.n_w), new(spec.n_w), new(spec.n_w), new(norm.n_w), new(norm.n_b)
    b.gated_forward(da, dWg, dWu, W_, bg=dbg, bu=dbu)
    b.conv_forward(plan, dx, dy, W_, z_, graph[0], graph[1])
    b.norm_forward(norm, z_, dw, dbias, y_, st, ptr=dptr)
    b.norm_backward(norm, z_, dw, dbias, dgy, st, gz, gw, gb, ptr=dptr)
    b.conv_backward(plan, dx, dy, W_, gz, gx, gye, gW, *graph)
    b.gated_backward(da, dWg, dWu, gW, ga, gWg, gWu, bg=dbg, bu=dbu, gbg=gbg, gbu=gbu)
    torch.cuda.synchronize()

    def near(got, ref, what):
        got = got.cpu().numpy().astype(np.float64)
        rms = np.sqrt(np.mean(ref ** 2))
        e = np.max(np.abs(got - ref) / np.maximum(np.abs(ref), rms))
        assert e <= tol, (what, e)

    near(y_, lay(n0["y"][0], "y"), "y")
    near(gx, lay(rx, "x"), "gx")
    near(gye, ry, "gy")
    near(gw, n0["gweight"][0], "gweight")
    near(gb, n0["gbias"][0], "gbias")
    for name, t in (("gx", ga), ("gWg", gWg), ("gWu", gWu), ("gbg", gbg), ("gbu", gbu)):
        near(t, rg[name][0], "gated " + name)
