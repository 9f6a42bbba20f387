"""What the entry points of the products by kind of row and of the orthogonalised updates refuse, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2501_13986_amd import binding as b

P = 256   # an aligned address that no refused call reaches


def forward(x=P, W=P, bias=0, out=P, rows=4, k=8, n=16, comps=1, groups=3, ptr=P, perm=0, ldx=8, ldo=16, dtype=0):
    return b.lib().grouped_forward(x, W, bias, out, rows, k, n, comps, groups, ptr, perm, ldx, ldo, dtype, None)


BOTH = [
    (dict(x=0), 1), (dict(W=0), 1), (dict(ptr=0), 1), (dict(x=P + 2), 1), (dict(W=P + 1), 1), (dict(ptr=P + 4), 1), (dict(perm=P + 4), 1),
    (dict(x=P + 4, dtype=1), 1), (dict(rows=-1), 1), (dict(groups=-1), 1), (dict(k=0), 1), (dict(n=0), 1), (dict(comps=0), 1), (dict(comps=-2), 1),
    (dict(ldx=7), 1), (dict(comps=3, ldx=23, ldo=48), 1), (dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(rows=1 << 31), 2), (dict(rows=1 << 30, comps=2, ldx=16, ldo=32), 2),
    (dict(comps=1025, ldx=1 << 20, ldo=1 << 20), 2), (dict(groups=(1 << 24) + 1), 2), (dict(k=(1 << 20) + 1, ldx=1 << 21), 2),
    (dict(k=1 << 16, ldx=1 << 16, n=1 << 16, ldo=1 << 16), 2), (dict(ldx=1 << 31), 2)]


@pytest.mark.parametrize("change,want", BOTH + [(dict(out=0), 1), (dict(out=P + 2), 1), (dict(ldo=15), 1), (dict(ldo=1 << 40), 2), (dict(bias=P + 2), 1), (dict(bias=P, comps=2, ldx=16, ldo=32), 1)])
def test_grouped_forward_refuses(change, want):
    assert forward(**change) == want
    assert b.lib().cgtp_last_error()


def test_grouped_without_rows_or_groups_launches_nothing():
    assert forward(rows=0) == 0 and forward(rows=0, x=0, out=0, ptr=0) == 0 and forward(groups=0, W=0, ptr=0) == 0
    assert backward(groups=0, W=0, gW=0, ptr=0) == 0


def backward(x=P, W=P, gout=P, gx=P, gW=P, gb=0, rows=4, k=8, n=16, comps=1, groups=3, ptr=P, perm=0, ldx=8, ldo=16, ldgx=8, dtype=0, ws=P, nws=1 << 40):
    return b.lib().grouped_backward(x, W, gout, gx, gW, gb, rows, k, n, comps, groups, ptr, perm, ldx, ldo, ldgx, dtype, ws, nws, None)


@pytest.mark.parametrize("change,want", BOTH + [(dict(gout=0), 1), (dict(gx=0), 1), (dict(gW=0), 1), (dict(gb=P + 2), 1), (dict(ldgx=7), 1), (dict(ldo=15), 1), (dict(ldgx=1 << 31), 2),
                                                (dict(gb=P, comps=2, ldx=16, ldo=32, ldgx=16), 1)])
def test_grouped_backward_refuses(change, want):
    change = dict({"ldgx": 1 << 21} if "ldgx" not in change else {}, **change)
    assert backward(**change) == want


def test_grouped_workspace():
    q = b.lib().cgtp_grouped_workspace_bytes
    assert q(0, 8, 16, 1, 3, 0) == 0 and q(4, 8, 16, 1, 0, 0) == 0 and q(-1, 8, 16, 1, 3, 0) == 0 and q(4, 0, 16, 1, 3, 0) == 0 and q(4, 8, 16, 1, 3, 5) == 0
    for rows in (1, 100, 3000, 160710):
        need = q(rows, 64, 96, 1, 20, 0)
        assert need % 256 == 0
        if need:
            assert backward(rows=rows, k=64, n=96, ldx=64, ldo=96, ldgx=64, groups=20, ws=0) == 1
            assert backward(rows=rows, k=64, n=96, ldx=64, ldo=96, ldgx=64, groups=20, ws=P + 128) == 1
            assert backward(rows=rows, k=64, n=96, ldx=64, ldo=96, ldgx=64, groups=20, nws=need - 1) == 1


COEFFICIENTS = (C.c_double * 6)(3, -4, 2, 3, -4, 2)
WIDE, TALL = dict(m=8, n=300, ldg=300, ldo=300, sg=2400, so=2400), dict(m=300, n=200, ldg=200, ldo=200, sg=60000, so=60000)      # sizes that need a workspace


def orth(g=P, out=P, batch=2, m=8, n=16, ldg=16, ldo=16, sg=128, so=128, c=COEFFICIENTS, steps=2, eps=1e-7, dtype=0, ws=P, nws=1 << 50):
    return b.lib().orthogonalise(g, out, batch, m, n, ldg, ldo, sg, so, c, steps, eps, dtype, ws, nws, None)


@pytest.mark.parametrize("change,want", [
    (dict(g=0), 1), (dict(out=0), 1), (dict(g=P + 2), 1), (dict(out=P + 4, dtype=1), 1), (dict(batch=-1), 1), (dict(m=0), 1), (dict(n=-1), 1),
    (dict(ldg=15), 1), (dict(ldo=15), 1), (dict(sg=-1), 1), (dict(so=-128), 1), (dict(so=127), 1), (dict(so=0), 1), (dict(so=8, ldo=20), 1), (dict(c=None), 1),
    (dict(c=(C.c_double * 6)(1, 2, 3, 4, float("nan"), 1)), 1), (dict(c=(C.c_double * 6)(1, 2, 3, 4, 1e39, 1)), 1), (dict(steps=0), 1), (dict(steps=65), 1), (dict(eps=0.0), 1),
    (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(eps=5e-324), 1), (dict(dtype=2), 1), (dict(WIDE, ws=0), 1), (dict(WIDE, ws=P + 128), 1), (dict(WIDE, nws=1), 1), (dict(TALL, ws=0), 1), (dict(TALL, nws=255), 1),
    (dict(batch=1 << 31), 2), (dict(m=1 << 16, n=1 << 16, ldg=1 << 16, ldo=1 << 16), 2), (dict(batch=1 << 30, m=1 << 10, n=1 << 10, ldg=1 << 10, ldo=1 << 10), 2), (dict(ldg=1 << 22), 2), (dict(ldo=1 << 50, so=1 << 59), 2), (dict(n=1 << 22, ldg=1 << 22, ldo=1 << 22), 2)])
def test_orthogonalise_refuses(change, want):
    assert orth(**change) == want
    assert b.lib().cgtp_last_error()


def test_orthogonalise_without_matrices_launches_nothing():
    assert orth(batch=0) == 0 and orth(batch=0, g=0, out=0) == 0
    assert b.lib().cgtp_orthogonalise_workspace_bytes(0, 8, 8, 0) == 0 and b.lib().cgtp_orthogonalise_workspace_bytes(2, 8, 0, 0) == 0


def refused(f, *a, **k):
    with pytest.raises(b.CgtpError) as e:
        f(*a, **k)
    return e.value.status == 1


def test_binding_refuses_tensors():
    x, W, out, ptr = torch.zeros(4, 8), torch.zeros(3, 8, 16), torch.zeros(4, 16), torch.zeros(4, dtype=torch.int64)
    call = lambda x=x, W=W, out=out, ptr=ptr, **k: refused(b.grouped_forward, x, W, out, ptr, **k)  # noqa: E731
    assert call()                                             # not on a GPU
    assert call(x=x.half()) and call(x=x.double()) and call(x=x[0]) and call(W=W[0]) and call(W=W[:, :7]) and call(out=out[:, :15]) and call(out=None)
    assert call(ptr=None) and call(ptr=ptr[1:]) and call(ptr=ptr.int()) and call(perm=ptr[1:]) and call(perm=torch.zeros(8, dtype=torch.int64)[::2])
    assert call(b=torch.zeros(3, 15)) and call(comps=0) and call(comps=2) and call(W=W.transpose(1, 2).contiguous().transpose(1, 2))
    back = lambda gout=out, gx=x, gW=W, **k: refused(b.grouped_backward, x, W, gout, gx, gW, ptr, **k)  # noqa: E731
    assert back() and back(gout=out[:, 1:]) and back(gx=None) and back(gW=W[:2]) and back(gb=torch.zeros(3, 8))
    G = torch.zeros(2, 4, 6)
    orth = lambda G=G, out=G, **k: refused(b.orthogonalise, G, out, **k)  # noqa: E731
    assert orth() and orth(G=G.half()) and orth(out=G[0]) and orth(out=None) and orth(G=G[0, 0]) and orth(G=G[0], out=None) and orth(out=G.double())
    assert orth(G=G.transpose(1, 2), out=torch.zeros(2, 6, 4)) and orth(coefficients=[(1.0, 2.0)])
