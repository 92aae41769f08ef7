"""A captured forward and backward pass replayed with other lengths in `starts`: which kernels run follows from the numbers of rows and sequences alone, and
each of them takes whatever lengths it finds."""
import pytest
import torch

from .test_gpu_attention import Attention

pytestmark = pytest.mark.gpu


def _other_lengths(total, n):
    """One long sequence and the rest short; all rows in the last; some rows in none; equal lengths."""
    yield [total - (n - 1)] + [1] * (n - 1)
    yield [0] * (n - 1) + [total]
    yield [max(0, total // n - 1)] * n
    yield [total // n] * n


@pytest.mark.parametrize("lengths,heads,kv_heads,dim,causal", [([20] * 120, 12, 12, 64, True), ([50] * 30, 2, 2, 128, False), ([90] * 20, 4, 2, 64, True),
                                                               ([700], 2, 1, 64, True), ([400] * 4, 8, 8, 96, False), ([9] * 70, 4, 4, 32, True)],
                         ids=lambda x: f"{len(x)}x{x[0]}" if isinstance(x, list) else str(x))
def test_replayed_with_other_lengths(lengths, heads, kv_heads, dim, causal):
    print("case replayed lengths", len(lengths), lengths[0], heads, kv_heads, dim, causal, flush=True)
    a = Attention(lengths, heads, kv_heads, dim, causal, seed=dim)
    a.forward()
    a.backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.forward()
        a.backward()
    for other in [lengths, *_other_lengths(sum(lengths), len(lengths)), lengths]:
        starts = [0]
        for n in other:
            starts.append(starts[-1] + n)
        a.starts_host = starts
        a.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        for t in (a.o, a.lse, a.dq, a.dk, a.dv):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        a.check()
