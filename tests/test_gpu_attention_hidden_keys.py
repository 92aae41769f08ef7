"""Keys that a program hides by their scores: one channel of the queries against a channel of the keys that holds the type's lowest value, or one whose
product is past fp32's range, so that the scores are minus infinity.  A row that sees other keys too has the results of those alone, wherever the hidden ones
stand: as all of the first tiles that its wave walks, too.  A row that sees hidden keys only, of equal finite scores, has their mean, and adds nothing to any
gradient: P = exp(S - lse) cannot be had from an lse of that size.

Bounds: the oracle's for the other keys alone.  The mean of n rows: weights of exactly 1, at most n roundings of 2^-24 of the mean of |v|, one to bf16 (2^-8 of
itself) and one of 2^-24 each for the total, its reciprocal and the product.  Such a row's lse is the score, of which log n is less than fp32 shows: a few
roundings, 2^-21 of itself."""
import pytest
import torch

from oracle import attention as oa

from .test_gpu_attention import Attention

pytestmark = pytest.mark.gpu

BATCHES = [([198], 2, 2, 64), ([198] * 180, 8, 8, 64), ([60] * 300, 8, 8, 64), ([60] * 300, 8, 8, 128), ([150] * 40, 8, 2, 64), ([90, 140] * 12, 6, 2, 128),
           ([1200] * 2, 24, 8, 64), ([1200, 700], 24, 24, 128), ([2100], 2, 1, 128)]


def _hidden(n):
    return n // 3 * 2 if n < 100 else n - 70


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("query,key,scale", [(1.0, -torch.finfo(torch.bfloat16).max, 0.125), (1.0, -torch.finfo(torch.bfloat16).max, 1.0),
                                             (2.0 ** 64, -2.0 ** 70, 0.125)], ids=["lowest", "lowest, past the range in base 2", "minus infinity"])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim", BATCHES, ids=lambda x: f"{len(x)}x{x[0]}" if isinstance(x, list) else str(x))
def test_hidden_keys(lengths, heads, kv_heads, dim, query, key, scale, causal):
    print("case hidden keys", len(lengths), lengths[0], heads, kv_heads, dim, query, key, scale, causal, flush=True)
    a = Attention(lengths, heads, kv_heads, dim, causal, seed=dim, scale=scale)
    for t, host, value in ((a.q, a.host[0], query), (a.k, a.host[1], 0.0)):
        t[:, :, 0] = value
        host[:, :, 0] = 0.0                                       # what the rows have of that channel where a key is not hidden
    spans = [(s, s + _hidden(n), s + n) for s, n in zip(a.starts_host, lengths)]
    for first, seen, _ in spans:
        a.k[first:seen, :, 0] = key
    a.forward()
    a.backward()
    got = a.outputs()
    q, k, v, do = (t.double() for t in a.host)
    finite = key * query * scale > -3.4e38
    for n, (first, seen, end) in enumerate(spans[:3] + spans[-1:]):
        rows = slice(seen if causal else first, end)              # causal: the rows before see hidden keys only
        for name, (value, bound) in oa.sequence(q[rows], k[seen:end], v[seen:end], scale, causal, do[rows]).items():
            if causal and not finite and name in ("dq", "dk", "dv"):
                continue                                          # next to rows that have no softmax
            x = {"lse": lambda: got["lse"][:, rows], "o": lambda: got["o"][rows], "dq": lambda: got["dq"][rows]}.get(name, lambda: got[name][seen:end])()
            if name == "dk":
                x, value, bound = x[:, :, 1:], value[:, :, 1:], bound[:, :, 1:]
            off = (x.double() - value).abs() / bound.clamp(min=1e-30)
            assert float(off.max()) <= 1.0, (name, n, float(off.max()))
        if finite or not causal:
            assert (got["dv"][first:seen] == 0).all() and (got["dk"][first:seen] == 0).all()
        if causal and finite:
            count = torch.arange(1, seen - first + 1).double()[:, None, None]
            vh = v[first:seen].repeat_interleave(heads // kv_heads, 1)
            mean, size = vh.cumsum(0) / count, vh.abs().cumsum(0) / count
            assert float(((got["o"][first:seen].double() - mean).abs() - (2.0 ** -8 * mean.abs() + (count + 3) * 2.0 ** -24 * size)).max()) <= 0
            assert float((got["lse"][:, first:seen].double() / (key * query * scale) - 1).abs().max()) <= 2.0 ** -21
            assert (got["dq"][first:seen] == 0).all()
        if causal and not finite:
            assert torch.isnan(got["o"][first:seen]).all()
