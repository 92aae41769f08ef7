"""Gradients of rows that see few keys: all of a sequence of up to 32 rows, the first 32 of a longer causal one.  Their delta = <do, o> carries no rounding of
o to bf16: a row of one key has no dq, whatever do is.

Bounds, with the oracle's e for a score and u = 4 e + 2^-20 for a softmax value (oracle.attention), g = (D + 1) 2^-24 sum |do| |v| for dP:
    delta = sum P dP is off by  sum P g + (u + 18 2^-24) sum P |dP|  (16 products in a lane, one sum of two lanes)
    dS    by  P (g + delta's) + (u + 2^-23) P (|dP| + |delta|), and 2^-8 |dS| for its rounding
    dq, dk by scale times that and 40 2^-24 |dS| (32 products, the factor) against |k|, |q|, and 2^-8 of themselves."""
import pytest
import torch

from .test_gpu_attention import Attention

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -8


def _gradients(q, k, v, do, scale, causal):
    """dq and dk of a sequence in float64 and their bounds."""
    group, D = q.shape[1] // k.shape[1], q.shape[2]
    q, k, v, do = (t.transpose(0, 1) for t in (q, k.repeat_interleave(group, 1), v.repeat_interleave(group, 1), do))
    S = scale * q @ k.transpose(1, 2)
    e = (D + 4) * 2.0 ** -24 * scale * q.abs() @ k.abs().transpose(1, 2)
    if causal:
        later = torch.ones(S.shape[1:], dtype=torch.bool).triu(1)
        S, e = S.masked_fill(later, float("-inf")), e.masked_fill(later, 0.0)
    P = torch.softmax(S, 2)
    u = 4 * e.amax(2, keepdim=True) + 2.0 ** -20
    dP, g = do @ v.transpose(1, 2), (D + 1) * 2.0 ** -24 * do.abs() @ v.abs().transpose(1, 2)
    delta = (P * dP).sum(2, keepdim=True)
    delta_off = (P * g).sum(2, keepdim=True) + (u + 18 * 2.0 ** -24) * (P * dP.abs()).sum(2, keepdim=True)
    dS = P * (dP - delta)
    off = P * (g + delta_off) + (u + 2.0 ** -23) * P * (dP.abs() + delta.abs()) + (STEP + 40 * 2.0 ** -24) * dS.abs()
    dq, dq_off = scale * dS @ k, scale * off @ k.abs()
    dk, dk_off = scale * dS.transpose(1, 2) @ q, scale * off.transpose(1, 2) @ q.abs()
    dk, dk_off = (t.reshape(-1, group, *t.shape[1:]).sum(1) for t in (dk, dk_off))
    return {"dq": (dq.transpose(0, 1), (dq_off + STEP * dq.abs()).transpose(0, 1)), "dk": (dk.transpose(0, 1), (dk_off + STEP * dk.abs()).transpose(0, 1))}


def _near(got, want, what):
    value, bound = want
    off = (got.double() - value).abs() / bound.clamp(min=1e-30)
    assert float(off.max()) <= 1.0, (what, float(off.max()))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (4, 2, 64), (3, 3, 32), (4, 1, 128), (2, 2, 128), (2, 2, 96)])
@pytest.mark.parametrize("lengths", [[1], [1, 2, 1, 3, 1], [32, 31, 5, 1], [1] * 300 + [17] * 40, [2, 9, 30, 14] * 90], ids=lambda n: f"{len(n)}x{n[0]}")
def test_short_sequences(lengths, heads, kv_heads, dim, causal):
    print("case few keys", len(lengths), lengths[0], heads, kv_heads, dim, causal, flush=True)
    a = Attention(lengths, heads, kv_heads, dim, causal, seed=dim + len(lengths))
    a.forward()
    a.backward()
    a.check()
    got = a.outputs()
    q, k, v, do = (t.double() for t in a.host)
    for first, n in list(zip(a.starts_host, lengths))[-60:]:
        rows = slice(first, first + n)
        want = _gradients(q[rows], k[rows], v[rows], do[rows], a.scale, causal)
        for name in want:
            _near(got[name][rows], want[name], (name, first, n))


@pytest.mark.parametrize("lengths,heads,kv_heads,dim", [([700], 2, 2, 64), ([700], 2, 1, 128), ([1500, 1300], 24, 24, 64), ([1500] * 3, 24, 8, 128), ([200] * 6, 4, 4, 64),
                                                        ([150] * 200, 8, 8, 64), ([90] * 40, 8, 2, 64)],
                         ids=lambda x: f"{len(x)}x{x[0]}" if isinstance(x, list) else str(x))
def test_the_first_rows_of_causal_sequences(lengths, heads, kv_heads, dim):
    print("case first rows", len(lengths), lengths[0], heads, kv_heads, dim, flush=True)
    a = Attention(lengths, heads, kv_heads, dim, True, seed=dim)
    a.forward()
    a.backward()
    got = a.outputs()
    q, k, v, do = (t.double() for t in a.host)
    for first in a.starts_host[:-1][:3] + a.starts_host[-2:-1]:
        rows = slice(first, first + 32)
        _near(got["dq"][rows], _gradients(q[rows], k[rows], v[rows], do[rows], a.scale, True)["dq"], first)
