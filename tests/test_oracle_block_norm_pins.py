"""The block norm oracle against a library routine, closed forms and differences."""
import pytest
import torch

from oracle import block_norm as ob


def _rand(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed + 31 * len(shape) + shape[0]))


def test_layer_norm_is_the_library_routines():
    z, w, b = _rand(5, 9), _rand(9), _rand(9, seed=1)
    torch.testing.assert_close(ob.norm(z, "layer", 1e-5, w, b), torch.nn.functional.layer_norm(z, (9,), w, b, 1e-5))


def test_rms_norm_of_a_constant_row_is_its_sign():
    z = torch.full((1, 6), -3.0, dtype=torch.float64)
    torch.testing.assert_close(ob.norm(z, "rms", 0.0, None, None), torch.full_like(z, -1.0))


@pytest.mark.parametrize("post,pre", [("none", "layer"), ("layer", "rms"), ("rms", "none"), ("rms", "layer")])
def test_gradients_against_differences(post, pre):
    x, h, gate, w2, b2, w1, b1 = _rand(3, 7), _rand(3, 7, seed=2), _rand(7, seed=3), _rand(7, seed=4), _rand(7, seed=5), _rand(7, seed=6), _rand(7, seed=7)
    dy, dn = _rand(3, 7, seed=8), _rand(3, 7, seed=9)

    def loss(x, h, gate, w2, b2, w1, b1):
        y, n, _ = ob.forward(x, h, gate, post, pre, 1e-5, 0.9, 0.7, w2, b2, w1, b1)
        return (y * dy).sum() + (0.0 if n is None else (n * dn).sum())

    leaves = [x, h, gate, w2, b2, w1, b1]
    y, _, _ = ob.forward(x, h, gate, post, pre, 1e-5, 0.9, 0.7, w2, b2, w1, b1)
    got = ob.backward(dy, dn if pre != "none" else None, h, y, gate, post, pre, 1e-5, 0.9, 0.7, w2, b2, w1)
    got["dgate"] = got["dgate"].sum(0)
    for n, name in enumerate(("dx", "dh", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")):
        if name not in got:
            continue
        for at in range(0, leaves[n].numel(), 3):
            d = torch.zeros_like(leaves[n]).flatten()
            d[at] = 1e-6
            up, down = list(leaves), list(leaves)
            up[n], down[n] = leaves[n] + d.view_as(leaves[n]), leaves[n] - d.view_as(leaves[n])
            assert float((loss(*up) - loss(*down)) / 2e-6) == pytest.approx(float(got[name].flatten()[at]), rel=1e-6, abs=1e-8), name
