"""More rows of a token table than one launch has groups of lanes for: 2^26 with 64 lanes to a row."""
import pytest
import torch

import paper_2304_08480_amd as dl

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_more_rows_than_a_launch_has_groups_of_lanes():
    rows, d, V = (1 << 26) + 77, 392, 61
    if torch.cuda.mem_get_info()[0] < rows * d * 2 + (8 << 30):
        pytest.skip("no memory for 2^26 rows")
    # every row of a run of 61 has another id, some of them none of the table's: a row that is left out or taken for another shows
    ids = torch.arange(rows, dtype=torch.int32, device="cuda") % (V + 2) - 1
    table = (torch.arange(V, device="cuda")[:, None] + torch.arange(d, device="cuda")[None] % 7).to(BF)        # whole numbers that bf16 holds
    y = torch.full((rows + 1, d), -1.0, dtype=BF, device="cuda")
    shape = dl.DiscoEmbedding(rows=rows, vocabulary=V, places=0, d=d, id_bits=32, table_dtype=dl.DISCO_BF16, y_dtype=dl.DISCO_BF16, grad_dtype=dl.DISCO_F32,
                              scale=1.0)
    print("case embedding forward", rows, d, flush=True)
    dl.disco_embedding_fwd(shape, ids, None, table, None, y, torch.cuda.current_stream())
    torch.cuda.synchronize()
    padded = torch.cat([torch.zeros_like(table[:1]), table, torch.zeros_like(table[:1])])
    period, step = len(padded), len(padded) << 15
    for at in range(0, rows, step):
        n = min(step, rows - at)
        assert torch.equal(y[at:at + n], padded.repeat((n + period - 1) // period, 1)[:n]), at
    assert bool((y[rows] == -1.0).all())
    # gradients of ones count the rows: below 2^24, so exact in any order
    y.fill_(1.0)
    need = dl.disco_embedding_workspace_bytes(shape)
    ws, grad = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.full((V, d), -1.0, device="cuda")
    print("case embedding backward", rows, d, flush=True)
    dl.disco_embedding_bwd(shape, ids, None, y, 0, grad, None, ws, need, torch.cuda.current_stream())
    torch.cuda.synchronize()
    count = torch.tensor([len(range(v + 1, rows, period)) for v in range(V)], device="cuda").float()
    assert torch.equal(grad, count[:, None].expand(V, d))
