"""Handles of the normalisation: every irreps string that the header accepts gives one, without a GPU."""
import pytest

from paper_2501_13986_amd import binding as b

# wide groups of several degrees: their code for registers is refused or relocates, so that the kernels for any size have to serve
WIDE = ["256x0e+256x1o+256x2e+256x3o+256x4e", "512x0e+512x1o+512x2e", "300x8e+300x7o+300x6e+300x5o+5000x0e"]


@pytest.mark.parametrize("flags", [b.CGTP_MUL_IR, b.CGTP_IR_MUL])
@pytest.mark.parametrize("dtype", [b.CGTP_F32, b.CGTP_F64])
@pytest.mark.parametrize("irreps", WIDE)
def test_wide_groups_have_kernels(irreps, dtype, flags):
    for act, gated in ((b.ACT_SILU, True), (b.ACT_TANH, False)):
        b.Norm(irreps, act=act, gated=gated, dtype=dtype, device=-2, flags=flags).close()
