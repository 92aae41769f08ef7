"""Plain float64 oracle of attention over packed sequences and of its gradients (test infrastructure only), written out from the definition,
with elementwise bounds on what bf16 softmax values and bf16 outputs may be off.

    S = scale q k^T (j <= i if causal), P = softmax(S), o = P v, lse = log sum exp S
    dv = P^T do, dP = do v^T, dS = P (dP - <do, o>), dq = scale dS k, dk = scale dS^T q (dk, dv summed over the heads that share the keys)

Bounds.  One rounding to bf16 is off by at most 2^-8 of the value.  A score is off by at most e = (D + 4) 2^-24 scale |q| |k| (a sum of D products in
fp32 and what is taken off it), a softmax value by about 2 e of itself (its own score and the total), here 4 e + 2^-20 with the exponential's and
the total's roundings.  So with u = 2^-8 + 4 e + 2^-20 for a softmax value that is rounded before it is multiplied:
    o    is off by  u sum P |v| + 2^-8 |o|
    dv   by         u sum P |do| + 2^-8 |dv|
    delta (from the stored o) by  sum |do| (o's bound);  dP by (D + 1) 2^-24 sum |do| |v|
    dS   by         P (those two) + u |dS|, and dq, dk by scale times that against |k|, |q|, + 2^-8 of themselves.
"""
from __future__ import annotations

import torch

STEP = 2.0 ** -8


def sequence(q, k, v, scale, causal, do=None):
    """One sequence: q L x H x D, k, v L x G x D in float64.  A dict of name -> (value, bound); lse H x L."""
    group = q.shape[1] // k.shape[1]
    D = q.shape[2]
    qh, kh, vh = (t.transpose(0, 1) for t in (q, k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)))
    S = scale * qh @ kh.transpose(1, 2)
    e = (D + 4) * 2.0 ** -24 * scale * qh.abs() @ kh.abs().transpose(1, 2)
    if causal:
        later = torch.ones(S.shape[1:], dtype=torch.bool).triu(1)
        S = S.masked_fill(later, float("-inf"))
        e = e.masked_fill(later, 0.0)
    e = e.amax(dim=2, keepdim=True)
    lse = torch.logsumexp(S, dim=2)
    P = torch.exp(S - lse[:, :, None])
    u = STEP + 4 * e + 2.0 ** -20
    o = P @ vh
    o_off = u * (P @ vh.abs()) + STEP * o.abs()
    out = {"o": (o, o_off), "lse": (lse, 2 * e[:, :, 0] + 2.0 ** -21 * (1 + lse.abs()))}
    if do is not None:
        dh = do.transpose(0, 1)
        dv = P.transpose(1, 2) @ dh
        dv_off = (u * P).transpose(1, 2) @ dh.abs() + 0.0
        dP = dh @ vh.transpose(1, 2)
        dS = P * (dP - (dh * o).sum(2, keepdim=True))
        off = (dh.abs() * o_off).sum(2, keepdim=True) + (D + 1) * 2.0 ** -24 * dh.abs() @ vh.abs().transpose(1, 2)
        dS_off = P * off + u * dS.abs()
        dq, dq_off = scale * dS @ kh, scale * dS_off @ kh.abs()
        dk, dk_off = scale * dS.transpose(1, 2) @ qh, scale * dS_off.transpose(1, 2) @ qh.abs()

        def shared(t):
            return t.reshape(k.shape[1], group, *t.shape[1:]).sum(1)

        dk, dk_off, dv, dv_off = shared(dk), shared(dk_off), shared(dv), shared(dv_off)
        for name, x, x_off in (("dq", dq, dq_off), ("dk", dk, dk_off), ("dv", dv, dv_off)):
            out[name] = (x, x_off + STEP * x.abs())
    return {name: x if name == "lse" else (x[0].transpose(0, 1), x[1].transpose(0, 1)) for name, x in out.items()}


def packed(q, k, v, starts, scale, causal, do=None):
    """All sequences; rows that belong to none are zeros with an infinite bound."""
    T = q.shape[0]
    like = {"o": q, "dq": q, "dk": k, "dv": v}
    out = {}
    for a, b in zip(starts[:-1], starts[1:]):
        if b <= a:
            continue
        got = sequence(q[a:b], k[a:b], v[a:b], scale, causal, None if do is None else do[a:b])
        for name, pair in got.items():
            if name not in out:
                shape = (q.shape[1], T) if name == "lse" else like[name].shape
                out[name] = (torch.zeros(shape, dtype=torch.float64), torch.full(shape, float("inf"), dtype=torch.float64))
            for x, y in zip(out[name], pair):
                if name == "lse":
                    x[:, a:b] = y
                else:
                    x[a:b] = y
    return out
