"""Handles of the normalisation: every irreps string that the header accepts gives one, without a GPU."""
import os
from concurrent.futures import ProcessPoolExecutor
from multiprocessing import get_context

import pytest

from paper_2501_13986_amd import binding as b
from perf.operators import IRREPS

# wide groups of several degrees: their code for registers is refused or relocates, so that the kernels for any size have to serve
WIDE = ["256x0e+256x1o+256x2e+256x3o+256x4e", "512x0e+512x1o+512x2e", "300x8e+300x7o+300x6e+300x5o+5000x0e"]


# so many segments that the compiler would leave calls in the kernels, with private memory for their arguments
MANY = "5000x0e+" + "+".join(["1x0e"] * 35)


def test_many_segments_have_kernels():
    b.Norm(MANY, act=b.ACT_NONE, device=-2).close()


@pytest.mark.parametrize("flags", [b.CGTP_MUL_IR, b.CGTP_IR_MUL])
@pytest.mark.parametrize("dtype", [b.CGTP_F32, b.CGTP_F64])
@pytest.mark.parametrize("irreps", WIDE)
def test_wide_groups_have_kernels(irreps, dtype, flags):
    for act, gated in ((b.ACT_SILU, True), (b.ACT_TANH, False)):
        b.Norm(irreps, act=act, gated=gated, dtype=dtype, device=-2, flags=flags).close()


def chosen(case):
    irreps, groups, act, dtype, flags = case
    n = b.Norm(irreps, groups=groups, act=act, dtype=dtype, device=-2, flags=flags)
    out = [n.kernel(ptr, backward) for ptr in (False, True) for backward in (False, True)]
    n.close()
    return out


REGISTERS = ["cgtp_norm_row_fwd", "cgtp_norm_row_bwd", "cgtp_norm_graph_fwd", "cgtp_norm_graph_bwd"]


@pytest.fixture
def pool(pytestconfig, monkeypatch, tmp_path):
    """Processes that compile side by side, their code kept between runs (a normalisation takes seconds to compile)."""
    kept = getattr(pytestconfig, "cache", None)
    monkeypatch.setenv("CGTP_CACHE_DIR", str(kept.mkdir("norm_kernels") if kept else tmp_path))
    with ProcessPoolExecutor(min(8, os.cpu_count() or 1), mp_context=get_context("spawn")) as p:
        yield p


def test_rows_of_the_models_are_held_in_registers(pool):
    """What this repository's convolutions put out, whatever the activation, layout and type.  (Room for private memory that no instruction uses
    once took small handles off these kernels: one graph of 20 000 rows 0.1 -> 4.3 ms.)"""
    cases = [(irreps, 1, act, dtype, flags) for irreps in IRREPS.values() for act in range(5) for dtype in (b.CGTP_F32, b.CGTP_F64)
             for flags in (b.CGTP_MUL_IR, b.CGTP_IR_MUL)]
    cases += [("4x0e+4x1o+4x1e+4x2e", 4, act, b.CGTP_F64, b.CGTP_IR_MUL) for act in range(5)]
    other = [(c, k) for c, k in zip(cases, pool.map(chosen, cases)) if k != REGISTERS]
    assert not other, other[:5]


def test_each_call_has_the_kernel_that_fits_it(pool):
    """A backward kernel that does not fit the registers takes no other one with it."""
    wide = [("512x0e+512x1o", b.CGTP_F32), ("2048x0e", b.CGTP_F32), ("1536x0e", b.CGTP_F32), ("1024x0e", b.CGTP_F64), ("256x0e+256x1o+256x2e+256x3o", b.CGTP_F64),
            ("384x0e+384x1o+384x2e+384x3o", b.CGTP_F32), ("8192x0e", b.CGTP_F32)]
    found = dict(zip(wide, pool.map(chosen, [(irreps, 1, b.ACT_SILU, dtype, b.CGTP_MUL_IR) for irreps, dtype in wide])))
    any_size = ["cgtp_norm_unit_fwd", "cgtp_norm_unit_bwd"] * 2
    assert found.pop(("8192x0e", b.CGTP_F32)) == any_size
    for case, k in found.items():
        assert (k[0], k[2]) == (REGISTERS[0], REGISTERS[2]), (case, k)
        assert all(got in pair for got, pair in zip(k, zip(REGISTERS, any_size))), (case, k)
    assert found[("512x0e+512x1o", b.CGTP_F32)][1] == REGISTERS[1]


def test_kernel_names_without_compiling():
    n = b.Norm("4x0e+4x1o", device=-1)
    assert [n.kernel(ptr, backward) for ptr in (False, True) for backward in (False, True)] == REGISTERS
    assert b.lib().cgtp_norm_kernel(None, 0, 0) is None


@pytest.mark.parametrize("irreps", ["8192x0e", "2048x0e", "65536x0e+65536x1o", "5000x0e+300x8e"])
def test_workspace_does_not_grow_with_the_samples(irreps):
    """Partial sums of the parameters' gradients are one row a workgroup, as many as fill the chip, not one a sample."""
    n = b.Norm(irreps, device=-2)
    assert n.kernel(False, True) == "cgtp_norm_unit_bwd"
    of = lambda N, S, ptr: b.lib().cgtp_norm_workspace_bytes(n._h, N, S, ptr, 1)  # noqa: E731
    row = 8 * (n.n_w + n.n_b)
    few = (256 << 20) + 256 * row + 256
    assert of(1_000_000, 1_000_000, 0) == of(50_000_000, 50_000_000, 0) <= few
    assert of(1_000_000, 40_000, 1) <= few and of(1000, 1, 1) <= row + 255 and of(3, 3, 0) <= 3 * row + 255
