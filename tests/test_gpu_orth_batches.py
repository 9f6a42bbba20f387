"""Orthogonalised updates in batches: what a matrix gives does not depend on the others where it has up to 128 rows or columns, and batches of several launches."""
import numpy as np
import pytest

from tests._products import orth_check
from tests.test_gpu_orth import gradients, run

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
PRECS = ["f32", "f64"]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("batch,m,n", [(5, 20, 30), (3, 64, 500), (9, 128, 128), (4, 301, 96), (7, 65, 70), (2, 10, 9000)])
def test_a_matrix_alone_gives_the_same_bits(batch, m, n, prec):
    G = gradients(batch, m, n, prec, seed=3)
    all_ = run(G)
    for i in (0, batch // 2, batch - 1):
        assert np.array_equal(run(G[i:i + 1])[0], all_[i])


@pytest.mark.parametrize("prec", PRECS)
def test_more_matrices_than_a_launch_has_workgroups(prec):
    from paper_2501_13986_amd import binding as b
    batch, edge = (1 << 22) + 40, 1 << 22
    t = torch.randn(batch, 2, 3, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.float32 if prec == "f32" else torch.float64)
    out = torch.full_like(t, float("nan"))
    b.orthogonalise(t, out)
    torch.cuda.synchronize()
    assert not torch.isnan(out).any()
    for at in (slice(0, 100), slice(edge - 50, edge + 40)):
        orth_check(out[at].cpu().numpy(), t[at].cpu().numpy(), prec, at)
    half = torch.empty_like(t[:batch // 2])
    for at in (slice(0, batch // 2), slice(batch - batch // 2, batch)):
        b.orthogonalise(t[at], half)
        assert torch.equal(half, out[at])
