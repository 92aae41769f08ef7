"""Cross attention with keys that their scores hide, and queries to which all of their keys are hidden: by an infinite channel, by the type's lowest value, or by products past fp32's
range.  All results, gradients of queries and keys among them, are those without these rows, within the oracle's bounds for the others alone; the rows
themselves have none: gradients of 0, and for queries o = 0 and lse = -infinity."""
import pytest
import torch

from oracle import cross_attention as oc

from .test_gpu_cross_attention import Cross

pytestmark = pytest.mark.gpu
INF, LOWEST = float("inf"), -torch.finfo(torch.bfloat16).max
# lengths, heads, key/value heads: rows of a key head in one tile of 32; the keys in shares; tiles of one wave and of four; the queries in shares
BATCHES = [([3, 1], [40, 50], 2, 1), ([1], [7], 1, 1), ([3, 1], [3000, 50], 4, 2), ([40] + [2] * 30, [90] + [33, 5, 64] * 10, 2, 2), ([70, 5], [300, 33], 2, 1),
           ([64, 1], [5000, 70], 2, 2), ([200, 130], [128, 600], 4, 1), ([5000, 3], [64, 20], 2, 1)]


def _hide(n):
    """Of n keys: the first that a wave sees if there are others, one between and the last."""
    first = min(32, n // 2)
    return sorted({*range(first), first + (n - first) // 2, n - 1} - {first})


def _compare(c, kept_q, kept_k, q_starts, k_starts):
    torch.cuda.synchronize()
    got = {n: t.double() for n, t in c.outputs().items()}
    want = oc.packed(*(c.host[n][kept].double() for n, kept in (("q", kept_q), ("k", kept_k), ("v", kept_k))), q_starts, k_starts, c.scale, c.host["do"][kept_q].double())
    for name, (value, bound) in want.items():
        x = got[name].T if name == "lse" else got[name]
        value, bound = (value.T, bound.T) if name == "lse" else (value, bound)
        kept = kept_k if name in ("dk", "dv") else kept_q
        finite = torch.isfinite(value)
        assert torch.equal(x[kept][~finite], value[~finite]), name
        off = (x[kept] - value).abs()[finite] / bound[finite].clamp(min=1e-30)
        assert not off.numel() or float(off.max()) <= 1.0, (name, float(off.max()))           # a NaN is not <= 1
        others = torch.ones(len(x), dtype=torch.bool)
        others[kept] = False
        assert torch.equal(x[others], torch.full_like(x[others], -INF if name == "lse" else 0.0)), name


def _kept(starts, gone):
    keep, at = [], [0]
    for a, b, rows in zip(starts[:-1], starts[1:], gone):
        keep += [r for r in range(a, b) if r - a not in rows]
        at.append(len(keep))
    return torch.tensor(keep, dtype=torch.long), at


@pytest.mark.parametrize("longest", [True, False])
@pytest.mark.parametrize("query,key", [(1.0, -INF), (-1.0, INF), (1.0, LOWEST), (2.0 ** 64, -2.0 ** 70)], ids=["minus infinity", "infinity", "lowest", "past the range"])
@pytest.mark.parametrize("batch", BATCHES, ids=lambda b: f"{len(b[0])}x{b[0][0]}x{b[1][0]}")
@pytest.mark.parametrize("dim", [24, 64, 96, 128])
def test_hidden_keys(dim, batch, query, key, longest):
    print("case cross attention hidden keys", dim, batch[0][:2], batch[1][:2], query, key, longest, flush=True)
    c = Cross(*batch, dim, seed=dim, longest=longest)
    gone = [_hide(n) for n in batch[1]]
    for name, value in (("q", query), ("k", 0.0)):
        c.host[name][:, :, 5] = value
        getattr(c, name).copy_(c.host[name])
    for start, rows in zip(c.ks, gone):
        c.k[[start + r for r in rows], :, 5] = key
    c.forward()
    c.backward()
    keys, k_starts = _kept(c.ks, gone)
    _compare(c, torch.arange(c.qs[-1]), keys, c.qs, k_starts)


@pytest.mark.parametrize("batch", BATCHES, ids=lambda b: f"{len(b[0])}x{b[0][0]}x{b[1][0]}")
@pytest.mark.parametrize("dim", [64, 128])
def test_sequences_whose_keys_are_all_hidden(dim, batch):
    print("case cross attention all keys hidden", dim, batch[0][:2], batch[1][:2], flush=True)
    c = Cross(*batch, dim, seed=dim)
    gone = [range(n) if i % 2 == 0 else [] for i, n in enumerate(batch[1])]
    c.host["q"][:, :, 5] = 1.0
    c.q[:, :, 5] = 1.0
    for start, rows in zip(c.ks, gone):
        c.k[start:start + len(rows), :, 5] = -INF
    c.forward()
    c.backward()
    keys, k_starts = _kept(c.ks, gone)
    queries, q_starts = _kept(c.qs, [range(n) if i % 2 == 0 else [] for i, n in enumerate(batch[0])])
    _compare(c, queries, keys, q_starts, k_starts)


@pytest.mark.parametrize("query", [-INF, INF])
@pytest.mark.parametrize("batch", BATCHES, ids=lambda b: f"{len(b[0])}x{b[0][0]}x{b[1][0]}")
@pytest.mark.parametrize("dim", [64, 128])
def test_queries_that_hide_all_keys(dim, batch, query):
    print("case cross attention blind queries", dim, batch[0][:2], batch[1][:2], query, flush=True)
    c = Cross(*batch, dim, seed=dim)
    gone = [sorted({0, n // 2, n - 1}) if n > 1 else [] for n in batch[0]]
    c.host["k"][:, :, 5] = 1.0 if query < 0 else -1.0
    c.k[:, :, 5] = c.host["k"][:, :, 5].cuda()
    for start, rows in zip(c.qs, gone):
        c.q[[start + r for r in rows], :, 5] = query
    c.forward()
    c.backward()
    queries, q_starts = _kept(c.qs, gone)
    _compare(c, queries, torch.arange(c.ks[-1]), q_starts, c.ks)


def test_what_is_no_number_is_not_taken_for_hidden():
    # NaN in a key's channel, and an infinite one that a query meets with 0, are NaN in the gradients of what sees them
    for k in (40, 3000):
        for value in (float("nan"), INF):
            c = Cross([3, 2], [k, 33], 2, 2, 64)
            c.q[:, :, 5] = 0.0
            c.k[k - 2, :, 5] = value
            c.forward()
            c.backward()
            assert torch.isnan(c.dq[:3]).all() and torch.isfinite(c.dq[3:]).all() and torch.isnan(c.dk[:k]).any() and torch.isfinite(c.dk[k:]).all()
