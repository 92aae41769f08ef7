"""One query over nearly 2^31 keys, where the keys with a score of 0 weigh in the softmax as the one that stands out does: a share of the keys that is lost or taken twice shows.

Keys and values are one buffer: zeros, and elevens in the last row.  The query is twos, so with 8 channels and a scale of 1/8 the last score is 22, the others 0, and
    Z = e^22 + n,  P = e^22 / Z of the last key (0.63) and 1 / Z of the others,  o = 11 P,  lse = log Z;  with do = 1:
    dv = P,  dS = P (dP - <do, o>) with dP = 88 of the last key and 0 of the others,  dk = dS q / 8,  dq = 11 dS / 8 of the last.
A share of 2^21 keys lost moves lse by 2^-10 n / Z = 3.7e-4, fifty times what it may be off.

Bounds.  Scores are exact, sums of ones exact within a share.  A weight e^-22 is off by 2^-23 of its exponent in base 2, 2.7e-6 of itself, the sum over 1024 shares (8 groups of 128) by
136 roundings of 2^-24, 8.2e-6, of n / Z = 0.37 of Z; so lse by 4.1e-6 with two roundings of 2^-24 of 22 and one of the logarithm's, 2^-22: below 2^-17 = 7.6e-6.
P backward, exp2 of a difference of up to 33 in base 2, off by 2^-23 of either: 2^-17 with lse's.  o, dv: 2^-8 of themselves for the type, o again 2^-8 for P's.  dS: <do, o> from o as
stored, 2^-7 of it, and 2^-8 for its own rounding."""
import math

import pytest
import torch

import paper_2304_08480_amd as dl

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_keys_that_weigh_together_as_much_as_one():
    tokens, dim, first = 2147483391, 8, 1000
    if torch.cuda.mem_get_info()[0] < 3 * tokens * dim * 2 + (8 << 30):
        pytest.skip("no memory for 2^31 keys and their gradients")
    buffer = torch.zeros(tokens, dim, dtype=BF, device="cuda")
    buffer[-1] = 11.0
    buffer[:first] = float("nan")                                       # rows of no sequence
    q, do = torch.full((1, 1, dim), 2.0, dtype=BF, device="cuda"), torch.ones(1, 1, dim, dtype=BF, device="cuda")
    o, dq, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(1, 1, device="cuda")
    dk, dv = (torch.full_like(buffer, -1.0) for _ in range(2))
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([first, tokens], dtype=torch.int32, device="cuda")
    shape = dl.DiscoCrossAttention(q_tokens=1, k_tokens=tokens, sequences=1, q_longest=1, k_longest=0, heads=1, kv_heads=1, head_dim=dim, dtype=dl.DISCO_BF16,
                                   scale=0.125, **{m + "_" + way: dim for m in "qkvo" for way in ("row", "head")})
    need = dl.disco_cross_attention_workspace_bytes(shape)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    print("case many keys, forward", flush=True)
    dl.disco_cross_attention_fwd(shape, *starts, q, buffer, buffer, o, lse, ws, need, torch.cuda.current_stream())
    torch.cuda.synchronize()
    n, e = tokens - first - 1, math.exp(22.0)
    z = n + e
    assert abs(float(lse) - math.log(z)) <= 2.0 ** -17 < (math.log(z) - math.log(z - 2 ** 21)) / 40
    assert float((o.double() / (11 * e / z) - 1).abs().max()) <= 2 * 2.0 ** -8 + 2.0 ** -16
    print("case many keys, backward", flush=True)
    dl.disco_cross_attention_bwd(shape, *starts, q, buffer, buffer, o, lse, do, dq, dk, dv, ws, need, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for t in (dk, dv):
        assert bool((t[:first] == -1.0).all())
    p, delta = e / z, 88 * e / z
    last = p * (88 - delta)
    off = p * delta * 2 * 2.0 ** -8 + last * (2.0 ** -8 + 2.0 ** -16)
    assert float((dv[-1].double() / p - 1).abs().max()) <= 2 * 2.0 ** -8 + 2.0 ** -16
    assert float((dk[-1].double() - last / 4).abs().max()) <= off / 4 + 2.0 ** -8 * last / 4
    assert float((dq.double() - last * 11 / 8).abs().max()) <= off * 11 / 8 + 2.0 ** -8 * last * 11 / 8
    for t, want, near in ((dv, 1 / z, 2 * 2.0 ** -8), (dk, -delta / z / 4, 4 * 2.0 ** -8)):
        assert abs(float(t[first, 0]) / want - 1) <= near + 2.0 ** -16
        for at in range(first, tokens - 1, 1 << 28):
            assert bool((t[at:min(at + (1 << 28), tokens - 1)] == t[first, 0]).all()), at
