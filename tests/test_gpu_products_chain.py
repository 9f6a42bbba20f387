"""A step of training of one matrix for each species, as a program makes it: rows sorted by species on the GPU, the layer forward and backward, the
update of the matrices orthogonalised."""
import numpy as np
import pytest

from oracle import products
from tests._products import check, grouped_tolerance, orth_check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("comps", [1, 3])
def test_sort_products_gradients_update(comps, prec):
    from paper_2501_13986_amd import binding as b
    rng = np.random.default_rng(comps)
    rows, species, K, n, dt = 400, 9, 24, 32, np.float32 if prec == "f32" else np.float64
    draw = lambda *s: rng.normal(size=s).astype(dt)  # noqa: E731
    kinds = rng.choice(species, rows, p=[0.5, 0, 0.2, 0.1, 0.1, 0, 0.05, 0.03, 0.02])
    x, W, target = draw(rows, comps * K), draw(species, K, n) / 5, draw(rows, comps * n)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    ptr, _, perm, _, _ = b.cgtp_csr_from_coo(dev(kinds.astype(np.int64)), torch.zeros(rows, dtype=torch.int64, device="cuda"), species if species > 1 else 1)
    dx, dW = dev(x), dev(W)
    out, gx, gW = dev(np.zeros_like(target)), torch.empty_like(dx), torch.empty_like(dW)
    b.grouped_forward(dx, dW, out, ptr, perm=perm, comps=comps)
    gout = out - dev(target)
    b.grouped_backward(dx, dW, gout, gx, gW, ptr, perm=perm, comps=comps)
    update = torch.empty_like(gW)
    b.orthogonalise(gW, update)
    torch.cuda.synchronize()

    order = np.argsort(kinds, kind="stable")
    assert np.array_equal(perm.cpu().numpy(), order)
    cuts = np.searchsorted(kinds[order], np.arange(species + 1))
    assert np.array_equal(ptr.cpu().numpy(), cuts)
    ref = products.grouped(x, W, cuts, order, None, comps, gout.cpu().numpy())
    for name, got, terms in (("out", out, K), ("gx", gx, n), ("gW", gW, rows * comps)):
        check(got.cpu().numpy(), ref[name], grouped_tolerance(ref[name], prec, terms), name)
    orth_check(update.cpu().numpy(), gW.cpu().numpy(), prec, "update")
    assert not update[1].any() and not update[5].any()      # species that were not seen
