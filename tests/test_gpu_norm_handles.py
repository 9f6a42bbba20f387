"""The normalisation of every kind of handle against the fp64 oracle: groups that registers do not hold."""
import pytest

from oracle import layer
from tests.test_gpu_norm import compare, handle, inputs, run
from tests.test_layer_handles import WIDE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", ["f32", "f64"])
@pytest.mark.parametrize("ir_mul", [False, True])
@pytest.mark.parametrize("irreps", WIDE)
def test_wide_groups(irreps, ir_mul, prec):
    for act, gated in ((layer.SILU, True), (layer.TANH, False)):
        n = handle(irreps, 1, act, gated, prec, ir_mul)
        for ptr in (None, [0, 5, 5, 11], [2, 12]):
            p = inputs(n, 12, prec, seed=3)
            compare(run(n, p, ptr), irreps, 1, act, gated, ir_mul, p, prec, ptr)
