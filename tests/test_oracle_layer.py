"""The oracle of the layer operators: gradients against differences, and what the definitions promise."""
import numpy as np
import pytest

from oracle import layer, so3
from oracle.irreps import parse_irreps

ACTS = [layer.NONE, layer.SILU, layer.GELU, layer.SIGMOID, layer.TANH]


def difference(f, x, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("kind", ACTS)
def test_activation_derivatives(kind):
    t = np.linspace(-6, 6, 41)
    a, d = layer.act(t, kind)
    assert np.allclose(d, (layer.act(t + 1e-5, kind)[0] - layer.act(t - 1e-5, kind)[0]) / 2e-5, atol=1e-8)
    assert np.abs(d).max() <= 1.13


@pytest.mark.parametrize("kind", ACTS)
def test_gated_gradients_are_the_differences(kind):
    rng = np.random.default_rng(3)
    p = [rng.normal(size=s) for s in ((3, 4), (4, 5), (4, 5), (5,), (5,))]
    t = rng.normal(size=(3, 5))
    ref = layer.gated(*p, kind, t)
    for i, name in enumerate(("gx", "gWg", "gWu", "gbg", "gbu")):
        f = lambda v: (layer.gated(*[v if j == i else q for j, q in enumerate(p)], kind)["out"][0] * t).sum()  # noqa: E731
        assert np.allclose(ref[name][0], difference(f, p[i]), atol=1e-7), name


NORMS = [("2x0e+2x1o+2x0o", 1, True, None), ("4x0e+2x2e", 2, True, [0, 1, 1, 4]), ("2x1e+2x0e", 1, False, [1, 3]), ("2x0e", 2, True, None)]


@pytest.mark.parametrize("irreps,groups,gated,ptr", NORMS)
@pytest.mark.parametrize("ir_mul", [False, True])
def test_norm_gradients_are_the_differences(irreps, groups, gated, ptr, ir_mul):
    rng = np.random.default_rng(5)
    segs, dx, dy = layer.norm_segments(irreps, gated)
    nw = sum(s[0] * (2 if s[5] >= 0 else 1) for s in segs)
    nb = sum(s[0] for s in segs if s[2] or s[5] >= 0)
    p = [rng.normal(size=s) for s in ((4, dx), (nw,), (nb,))]
    t = rng.normal(size=(4, dy))
    run = lambda q, g=None: layer.norm(irreps, groups, layer.SILU, gated, 1e-2, ir_mul, *q, ptr, g)  # noqa: E731
    ref = run(p, t)
    own = ~np.isnan(ref["y"][0])
    assert own.all(1).tolist() == [ptr is None or ptr[0] <= r < ptr[-1] for r in range(4)]
    for i, name in enumerate(("gx", "gweight", "gbias")):
        f = lambda v: (run([v if j == i else q for j, q in enumerate(p)])["y"][0][own] * t[own]).sum()  # noqa: E731
        got = ref[name][0]
        assert np.allclose(np.nan_to_num(got), difference(f, p[i]), atol=1e-6), name


def test_norm_is_equivariant():
    """Rotated rows give rotated results: no segment but 0e is shifted, and what multiplies it does not depend on the frame."""
    irreps = "3x0e+2x1o+2x2e"
    rng = np.random.default_rng(1)
    segs, dx, dy = layer.norm_segments(irreps, True)
    x, w, b = rng.normal(size=(4, dx)), rng.normal(size=11), rng.normal(size=7)
    D = {l: so3.wigner_D_real(l, 0.3, 1.1, -0.7) for l in range(3)}

    def turned(v):
        v, at = v.copy(), 0
        for ir in parse_irreps(irreps):
            n = 2 * ir.l + 1
            for u in range(ir.mul):
                v[:, at:at + n] = v[:, at:at + n] @ D[ir.l].T
                at += n
        return v

    run = lambda v: layer.norm(irreps, 1, layer.SILU, True, 1e-5, False, v, w, b, [0, 3, 4])["y"][0]  # noqa: E731
    assert np.allclose(run(turned(x)), turned(run(x)), atol=1e-12)


def test_norm_statistics():
    x = np.random.default_rng(0).normal(size=(6, 8)) * 3 + 2
    r = layer.norm("4x0e+2x0o", 2, layer.NONE, True, 1e-300, False, x, np.ones(8), np.zeros(6), [0, 6])["y"][0]
    for g in range(2):
        v = r[:, 2 * g:2 * g + 2]
        assert abs(v.mean()) < 1e-12 and abs((v ** 2).mean() - 1) < 1e-12
