"""The attention oracle against closed forms, autograd and differences."""
import pytest
import torch

from oracle import attention as oa


def _case(L=7, H=4, G=2, D=8, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(L, n, D, dtype=torch.float64, generator=g) for n in (H, G, G, H)]


def test_one_token_returns_its_value_and_moves_only_it():
    q, k, v, do = _case(L=1)
    got = oa.sequence(q, k, v, 0.3, True, do)
    torch.testing.assert_close(got["o"][0], v.repeat_interleave(2, 1))
    torch.testing.assert_close(got["lse"][0][:, 0], 0.3 * (q * k.repeat_interleave(2, 1)).sum(2)[0])
    torch.testing.assert_close(got["dv"][0], do.reshape(1, 2, 2, 8).sum(2))
    assert float(got["dq"][0].abs().max()) < 1e-15 and float(got["dk"][0].abs().max()) < 1e-15


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_autograd_and_differences(causal):
    q, k, v, do = _case()
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]

    def loss(q, k, v):
        o = []
        for h in range(4):
            s = 0.4 * q[:, h] @ k[:, h // 2].T
            if causal:
                s = s.masked_fill(torch.ones(7, 7, dtype=torch.bool).triu(1), float("-inf"))
            o.append(s.softmax(1) @ v[:, h // 2])
        return (torch.stack(o, 1) * do).sum()

    want = torch.autograd.grad(loss(*leaves), leaves)
    got = oa.sequence(q, k, v, 0.4, causal, do)
    for name, w in zip(("dq", "dk", "dv"), want):
        torch.testing.assert_close(got[name][0], w)
    for n, (name, t) in enumerate(zip(("dq", "dk", "dv"), (q, k, v))):
        d = torch.zeros_like(t)
        d[3, 1, 2] = 1e-6
        up, down = [list((q, k, v)) for _ in range(2)]
        up[n], down[n] = t + d, t - d
        assert float((loss(*up) - loss(*down)) / 2e-6) == pytest.approx(float(got[name][0][3, 1, 2]), rel=1e-6, abs=1e-8)


def test_packed_rows_are_their_sequences():
    q, k, v, do = _case(L=12, seed=1)
    got = oa.packed(q, k, v, [1, 5, 5, 10], 0.2, True, do)
    one = oa.sequence(q[5:10], k[5:10], v[5:10], 0.2, True, do[5:10])
    for name in ("o", "dq", "dk", "dv"):
        torch.testing.assert_close(got[name][0][5:10], one[name][0])
        assert torch.isinf(got[name][1][0]).all() and torch.isinf(got[name][1][10:]).all()
    torch.testing.assert_close(got["lse"][0][:, 5:10], one["lse"][0])
