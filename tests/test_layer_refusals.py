"""What the entry points of the layer operators refuse, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2501_13986_amd import binding as b

P = 256   # an aligned address that no refused call reaches


def status(s):
    return {v: k for k, v in b.STATUS.items()}[s]


EINVAL, EUNSUPPORTED = status("CGTP_EINVAL"), status("CGTP_EUNSUPPORTED")


def forward(x=P, Wg=P, Wu=P, bg=0, bu=0, out=P, rows=4, k=8, n=16, ldx=8, ldo=16, act=1, dtype=0):
    return b.lib().gated_forward(x, Wg, Wu, bg, bu, out, rows, k, n, ldx, ldo, act, dtype, None)


@pytest.mark.parametrize("change,want", [
    (dict(x=0), 1), (dict(Wg=0), 1), (dict(Wu=0), 1), (dict(out=0), 1), (dict(x=P + 4), 1), (dict(out=P + 8), 1), (dict(Wu=P + 4), 1),
    (dict(bg=P), 1), (dict(bu=P), 1), (dict(rows=-1), 1), (dict(k=0), 1), (dict(n=0), 1), (dict(n=-3), 1), (dict(ldx=7), 1), (dict(ldo=15), 1),
    (dict(act=5), 1), (dict(act=-1), 1), (dict(dtype=2), 1), (dict(rows=1 << 31), 2), (dict(n=(1 << 20) + 1, ldo=1 << 21), 2), (dict(k=(1 << 20) + 1, ldx=1 << 21), 2),
    (dict(k=1 << 16, ldx=1 << 16, n=1 << 16, ldo=1 << 16), 2), (dict(ldx=1 << 22), 2), (dict(ldo=1 << 40), 2)])
def test_gated_forward_refuses(change, want):
    assert forward(**change) == want
    assert b.lib().cgtp_last_error()


def test_gated_without_rows_launches_nothing():
    assert forward(rows=0) == 0
    assert forward(rows=0, x=0, out=0) == 0


def backward(x=P, Wg=P, Wu=P, bg=0, bu=0, gout=P, gx=P, gWg=P, gWu=P, gbg=0, gbu=0, rows=4, k=8, n=16, ldx=8, ldg=16, ldgx=8, act=1, dtype=0,
             ws=P, nws=None):
    nws = b.lib().cgtp_gated_workspace_bytes(4, 8, 16, 0) if nws is None else nws
    return b.lib().gated_backward(x, Wg, Wu, bg, bu, gout, gx, gWg, gWu, gbg, gbu, rows, k, n, ldx, ldg, ldgx, act, dtype, ws, nws, None)


@pytest.mark.parametrize("change,want", [
    (dict(x=0), 1), (dict(gout=0), 1), (dict(gx=0), 1), (dict(gWg=0), 1), (dict(gWu=0), 1), (dict(gWu=P + 4), 1), (dict(bg=P, bu=P), 1),
    (dict(gbg=P, gbu=P), 1), (dict(bg=P, bu=P, gbg=P), 1), (dict(ldg=15), 1), (dict(ldgx=7), 1), (dict(ws=0), 1), (dict(ws=P + 128), 1),
    (dict(nws=1), 1), (dict(act=9), 1), (dict(dtype=7), 1), (dict(rows=1 << 31), 2)])
def test_gated_backward_refuses(change, want):
    assert backward(**change) == want


def test_gated_workspace_query():
    q = b.lib().cgtp_gated_workspace_bytes
    assert q(0, 8, 16, 0) == 0 and q(-1, 8, 16, 0) == 0 and q(4, 0, 16, 0) == 0 and q(4, 8, 16, 3) == 0
    sizes = [q(r, 64, 2176, 0) for r in (1, 2, 17, 100, 1000, 30000, 160710, 1 << 20)]
    assert all(s % 256 == 0 for s in sizes) and max(sizes) < 1 << 30


def make(irreps="4x0e+4x1o", groups=1, act=1, eps=1e-5, dtype=0, device=-1, flags=0):
    h = C.c_void_p()
    s = b.lib().cgtp_norm_create(irreps.encode() if irreps is not None else None, groups, act, eps, dtype, device, flags, C.byref(h))
    if s == 0:
        b.lib().cgtp_norm_destroy(h)
    else:
        assert not h
    return s


@pytest.mark.parametrize("change,want", [
    (dict(irreps=None), 1), (dict(irreps=""), 1), (dict(irreps="4x1q"), 1), (dict(irreps="0x1o"), 1), (dict(groups=0), 1), (dict(groups=3), 1),
    (dict(groups=-4), 1), (dict(act=5), 1), (dict(eps=0.0), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
    (dict(dtype=2), 1), (dict(flags=4), 1), (dict(irreps="2x9e"), 2), (dict(irreps="65537x0e"), 2), (dict(irreps="+".join(["1x0e"] * 65)), 2)])
def test_norm_create_refuses(change, want):
    assert make(**change) == want
    assert b.lib().cgtp_last_error()


def test_norm_eps_is_a_normal_number_of_its_type():
    """1e-40 would be zero for some fp32 arithmetic, 1 / sqrt(eps) infinite and a constant row NaN."""
    assert make(eps=1e-40) == 1 and make(eps=1e39) == 1 and make(eps=5e-324, dtype=b.CGTP_F64) == 1
    assert make(eps=2.0 ** -126) == 0 and make(eps=1e-40, dtype=b.CGTP_F64) == 0


def test_norm_dims():
    n = b.Norm("4x0e+3x1o+2x0o", groups=1, gated=True, device=-1)
    assert (n.dim_x, n.dim_y, n.n_w, n.n_b, n.n_stat) == (4 + 9 + 2 + 5, 15, 14, 9, 10)
    n = b.Norm("4x0e+4x1o", groups=2, gated=False, device=-1)
    assert (n.dim_x, n.dim_y, n.n_w, n.n_b, n.n_stat) == (16, 16, 8, 4, 8)
    assert b.lib().cgtp_norm_dim(n._h, 5) == -1 and b.lib().cgtp_norm_dim(None, 0) == -1


def test_norm_calls_refuse():
    n = b.Norm("4x0e+4x1o", device=-1)
    L = b.lib()
    fwd = lambda h=n._h, x=P, w=P, bi=P, y=P, st=P, N=3, S=3, ptr=0: L.norm_forward(h, x, w, bi, y, st, N, S, ptr, P, 1 << 30, None)  # noqa: E731
    assert fwd(h=None) == 1 and fwd(N=-1) == 1 and fwd(S=-1, ptr=P) == 1 and fwd(S=4) == 1 and fwd(x=P + 4) == 1
    assert fwd(N=1 << 31, S=1 << 31) == 2
    assert fwd() == 2          # made without a device
    assert b"not loaded" in L.cgtp_last_error()
    bwd = lambda N=3, S=3, gw=P: L.norm_backward(n._h, P, P, P, P, P, P, gw, P, N, S, 0, P, 1 << 30, None)  # noqa: E731
    assert bwd(N=-1) == 1 and bwd() == 2
    assert L.cgtp_norm_destroy(None) == 0


def test_norm_kernels_compile_without_a_gpu():
    for irreps, groups in (("32x0e+32x1o+32x2e+32x3o", 4), ("7x0e+5x1o+3x2e+9x0e", 1), ("1x8e", 1)):
        for dt in (b.CGTP_F32, b.CGTP_F64):
            b.Norm(irreps, groups=groups, dtype=dt, device=-2).close()


def refused(f, *a, **k):
    with pytest.raises(b.CgtpError) as e:
        f(*a, **k)
    return e.value.status == EINVAL


def test_binding_refuses_tensors():
    x, W, out = torch.zeros(4, 8), torch.zeros(8, 16), torch.zeros(4, 16)
    call = lambda x=x, Wg=W, Wu=W, out=out, **k: refused(b.gated_forward, x, Wg, Wu, out, **k)  # noqa: E731
    assert call()                                             # not on a GPU
    assert call(x=x.half()) and call(x=x.double()) and call(x=x[0]) and call(x=x.T.contiguous().T) and call(Wu=torch.zeros(8, 15))
    assert call(Wg=torch.zeros(16, 8).T) and call(out=torch.zeros(4, 32)[:, ::2]) and call(bg=torch.zeros(16)) and call(out=None)
    n = b.Norm("4x0e+4x1o", device=-1)
    rows, w, bias, y = torch.zeros(3, n.dim_x), torch.zeros(n.n_w), torch.zeros(n.n_b), torch.zeros(3, n.dim_y)
    norm = lambda x=rows, w=w, bias=bias, y=y, **k: refused(b.norm_forward, n, x, w, bias, y, **k)  # noqa: E731
    assert norm() and norm(x=rows.double()) and norm(x=rows[:, 1:]) and norm(w=w[1:]) and norm(bias=None) and norm(y=None)
    assert norm(ptr=torch.zeros(4)) and norm(ptr=torch.zeros(0, dtype=torch.int64)) and norm(stats=torch.zeros(5))
    assert norm(ptr=torch.zeros(8, dtype=torch.int64)[::2])
