"""The widest rows, whose workgroups have as many lanes as there are, with both norms and every kind of gate, in 16 bits, 32 and both."""
import pytest

from .test_gpu_block_norm import Norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,h", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("gate", ["none", "channel", "element"])
@pytest.mark.parametrize("rows,d", [(600, 4097), (37, 6000), (5, 8191), (600, 8192)])
def test_wide_rows(rows, d, gate, x, h):
    print("case block norm", rows, d, gate, x, h, flush=True)
    n = Norm(rows, d, "layer", "rms", gate, x, h, seed=d)
    n.forward()
    n.backward()
    n.check()
    one = n.outputs()
    n.backward()
    assert all((one[k] == v).all() for k, v in n.outputs().items())
