"""Token table with so many rows that its gradients' list is cut into longer pieces, in both tables, several blocks of columns, with and without accumulation.  All values are whole
numbers, halves after the scale, and all sums below 2^23: fp32 holds them exactly in whatever order, so every entry is compared for equality and a row that is lost or taken twice shows."""
import pytest
import torch

import paper_2304_08480_amd as dl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,d,bits", [((1 << 18) + 77, 8, 32), ((1 << 18) + 77, 600, 64), ((1 << 17) - 1, 1100, 32), ((1 << 20) + 3, 77, 32)])
def test_pieces_of_both_tables(rows, d, bits, accumulate):
    print("case embedding pieces", rows, d, bits, accumulate, flush=True)
    V, P = 40, 31
    whole = torch.int64 if bits == 64 else torch.int32
    g = torch.Generator(device="cuda").manual_seed(d)

    def numbers(*shape):
        return torch.randint(-4, 5, shape, generator=g, device="cuda").float()

    # frequent ids more often, some that neither table has
    ids = (V * torch.rand(rows, generator=g, device="cuda") ** 3).long() - 1
    place = torch.arange(rows, device="cuda") % (P + 3) - 1
    table, places, dy = numbers(V, d), numbers(P, d), numbers(rows, d)
    shape = dl.DiscoEmbedding(rows=rows, vocabulary=V, places=P, d=d, id_bits=bits, table_dtype=dl.DISCO_F32, y_dtype=dl.DISCO_F32, grad_dtype=dl.DISCO_F32,
                              scale=0.5)
    y = torch.full((rows + 1, d), -9.0, device="cuda")
    i, p = ids.to(whole), place.to(whole)
    dl.disco_embedding_fwd(shape, i, p, table, places, y, torch.cuda.current_stream())
    assert bool((y[rows] == -9.0).all())

    def there(x, n):
        return (x >= 0) & (x < n)

    want = torch.where(there(ids, V)[:, None], 0.5 * table[ids.clamp(0, V - 1)], 0.0) + torch.where(there(place, P)[:, None], places[place.clamp(0, P - 1)], 0.0)
    assert torch.equal(y[:rows], want)
    need = dl.disco_embedding_workspace_bytes(shape)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    old = [numbers(V, d), numbers(P, d)]
    grads = [t.clone() if accumulate else torch.full_like(t, float("nan")) for t in old]
    dl.disco_embedding_bwd(shape, i, p, dy, accumulate, *grads, ws, need, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for got, before, x, n, scale in zip(grads, old, (ids, place), (V, P), (0.5, 1.0)):
        kept = there(x, n)
        # sums of whole numbers: exact
        total = torch.zeros(n, d, dtype=torch.float64).index_add_(0, x[kept].cpu(), dy[kept].cpu().double())
        assert float(total.abs().max()) < 2 ** 23
        assert torch.equal(got.cpu().double(), scale * total + (before.cpu().double() if accumulate else 0.0))
