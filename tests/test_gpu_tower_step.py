"""A training step of a text tower around the loss, as a program runs it: packed captions, norm before the block, attention, gate, residual sum and last
norm, the captions' last tokens as features, their normalisation, the loss, everything backwards, the gradients clipped.

The reference walks the same chain with the float64 oracles and rounds to bf16 wherever the program stores bf16.  What is left between the two: a value
that lies on a rounding border for one of them and not for the other (in fp32's 2^-24, so for one of some 2^15 values), and the softmax values and their
gradients, which attention rounds to bf16 inside, once each pass: 2^-8 of the values that it adds up, twice in the gradients that have passed it (dq, dk
from dS; dS from the stored o).  Relative to a gradient's norm that is 3 x 2^-8 at most where all roundings fall the same way; the loss's own numerators
are bf16 too (2^-8).  4 x 2^-8 bounds every compared gradient.
"""
import numpy as np
import pytest
import torch

import paper_2304_08480_amd as dl
from oracle import attention as oa
from oracle import block_norm as ob
from oracle import clip_oracle as oc
from oracle import feature_prep as op

pytestmark = pytest.mark.gpu
EPS, S, WIDTH, HEADS, HEAD = 1e-5, 14.285714, 64, 4, 16
BOUND = 4 * 2.0 ** -8


def b(t):
    """As bf16 holds it, in float64."""
    return t.to(torch.bfloat16).double()


def _inputs(B):
    g = torch.Generator().manual_seed(B)

    def r(*shape, scale=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g) * scale).to(dtype)

    lengths = torch.randint(1, 30, (B,), generator=g).tolist()
    lengths[3] = 140                                      # one that the kernels for short sequences leave to the others
    starts = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    T = int(starts[-1])
    inner = HEADS * HEAD
    return {"starts": starts, "tokens": r(T, WIDTH), "places": r(T, WIDTH, scale=0.5), "w_qkv": r(3 * inner, WIDTH, scale=WIDTH ** -0.5),
            "w_out": r(WIDTH, inner, scale=inner ** -0.5), "gate": 1.0 + r(WIDTH, scale=0.1, dtype=torch.float32),
            "w0": 1.0 + r(WIDTH, scale=0.1, dtype=torch.float32), "b0": r(WIDTH, scale=0.1, dtype=torch.float32),
            "w1": 1.0 + r(WIDTH, scale=0.1, dtype=torch.float32), "b1": r(WIDTH, scale=0.1, dtype=torch.float32),
            "images": torch.nn.functional.normalize(torch.randn(B, WIDTH, generator=g), dim=1).to(torch.bfloat16)}


def _reference(x, max_norm):
    d = {k: v.double() for k, v in x.items() if k != "starts"}
    starts = x["starts"].tolist()
    T, inner, last = starts[-1], HEADS * HEAD, torch.from_numpy(x["starts"][1:].astype(np.int64) - 1)
    y0, n0, _ = ob.forward(d["places"], d["tokens"], None, "none", "layer", EPS, 1.0, 1.0, None, None, d["w0"], d["b0"], stored=b)
    y0, n0 = b(y0), b(n0)
    qkv = b(n0 @ d["w_qkv"].T)
    q, k, v = (t.reshape(T, HEADS, HEAD) for t in qkv.split(inner, 1))
    scale = HEAD ** -0.5
    o = b(oa.packed(q, k, v, starts, scale, True)["o"][0])
    p = b(o.reshape(T, inner) @ d["w_out"].T)
    y1, n1, _ = ob.forward(y0, p, d["gate"], "none", "layer", EPS, 1.0, 1.0, None, None, d["w1"], d["b1"], stored=b)
    y1, n1 = b(y1), b(n1)
    f = n1[last].numpy()
    u, inv = op.l2_normalize_fwd(f)
    u = b(torch.from_numpy(u)).numpy()
    loss, gI, gT, gs = oc.clip_loss_full(d["images"].numpy(), u, S)
    df = op.l2_normalize_bwd(gT, f)
    dn1 = torch.zeros(T, WIDTH, dtype=torch.float64)
    dn1[last] = b(torch.from_numpy(df))
    join = ob.backward(None, dn1, p, y1, d["gate"], "none", "layer", EPS, 1.0, 1.0, None, None, d["w1"])
    dy0, dp = b(join["dx"]), b(join["dh"])
    do = b(dp @ d["w_out"]).reshape(T, HEADS, HEAD)
    got = oa.packed(q, k, v, starts, scale, True, do)
    dqkv = torch.cat([b(got[n][0]).reshape(T, inner) for n in ("dq", "dk", "dv")], 1)
    dn0 = b(dqkv @ d["w_qkv"])
    first = ob.backward(dy0, dn0, d["tokens"], y0, None, "none", "layer", EPS, 1.0, 1.0, None, None, d["w0"])
    grads = {"w_qkv": dqkv.T @ n0, "w_out": dp.T @ o.reshape(T, inner), "gate": join["dgate"].sum(0), "w0": first["dw_pre"], "b0": first["db_pre"],
             "w1": join["dw_pre"], "b1": join["db_pre"], "tokens": b(first["dh"]), "places": b(first["dx"])}
    norm = float(torch.sqrt(sum((g ** 2).sum() for g in grads.values())))
    return float(loss), grads, norm


class Step:
    """The program's buffers and its step."""

    def __init__(self, x, B, max_norm):
        self.x = {k: (torch.from_numpy(v) if k == "starts" else v).cuda() for k, v in x.items()}
        self.B, self.max_norm = B, max_norm
        T, inner = int(x["starts"][-1]), HEADS * HEAD
        self.T, self.last = T, torch.from_numpy(x["starts"][1:].astype(np.int64) - 1).cuda()

        def e(*shape, dtype=torch.bfloat16):
            return torch.full(shape, float("nan"), dtype=dtype, device="cuda")

        f32 = torch.float32
        self.y0, self.n0, self.y1, self.n1, self.dy0, self.dp, self.dx, self.dh = (e(T, WIDTH) for _ in range(8))
        self.st0, self.st1 = e(T, 4, dtype=f32), e(T, 4, dtype=f32)
        self.o, self.lse, self.dqkv = e(T, HEADS, HEAD), e(HEADS, T, dtype=f32), e(T, 3 * inner)
        self.u, self.inv, self.df = e(B, WIDTH), e(B, dtype=f32), e(B, WIDTH, dtype=f32)
        self.loss, self.gs, self.gI, self.gT = e(1, dtype=f32), e(1, dtype=f32), e(B, WIDTH, dtype=f32), e(B, WIDTH, dtype=f32)
        self.dn1 = torch.zeros(T, WIDTH, dtype=torch.bfloat16, device="cuda")
        self.small = {k: e(WIDTH, dtype=f32) for k in ("gate", "w0", "b0", "w1", "b1")}
        self.norm = e(1, dtype=f32)
        bf, none, layer = dl.DISCO_BF16, dl.DISCO_NORM_NONE, dl.DISCO_NORM_LAYER
        shape = dict(rows=T, d=WIDTH, post=none, pre=layer, x_dtype=bf, h_dtype=bf, eps_pre=EPS, x_scale=1.0, h_scale=1.0)
        self.s0, self.s1 = dl.DiscoBlockNorm(gate=dl.DISCO_GATE_NONE, **shape), dl.DiscoBlockNorm(gate=dl.DISCO_GATE_CHANNEL, **shape)
        row = {m + "_row": 3 * inner for m in "qkv"} | {m + "_head": HEAD for m in "qkvo"} | {"o_row": inner}
        self.sa = dl.DiscoAttention(tokens=T, sequences=B, heads=HEADS, kv_heads=HEADS, head_dim=HEAD, causal=1, dtype=bf, scale=HEAD ** -0.5, **row)
        self.need = max(dl.disco_block_norm_workspace_bytes(self.s1), dl.disco_attention_workspace_bytes(self.sa), dl.disco_grad_workspace_bytes(9),
                        dl.disco_workspace_bytes(B, WIDTH, 1, bf, dl.DISCO_PATH_AUTO))
        self.ws = torch.full((self.need,), 255, dtype=torch.uint8, device="cuda")

    def run(self):
        x, T, inner, ws, need = self.x, self.T, HEADS * HEAD, self.ws, self.need
        s = torch.cuda.current_stream()
        bf = dl.DISCO_BF16
        dl.disco_block_norm_fwd(self.s0, x["places"], x["tokens"], None, None, None, x["w0"], x["b0"], self.y0, self.n0, self.st0, s)
        qkv = self.n0 @ x["w_qkv"].T
        q, k, v = (t.view(T, HEADS, HEAD) for t in qkv.split(inner, 1))
        dl.disco_attention_fwd(self.sa, x["starts"], q, k, v, self.o, self.lse, s)
        p = self.o.view(T, inner) @ x["w_out"].T
        dl.disco_block_norm_fwd(self.s1, self.y0, p, x["gate"], None, None, x["w1"], x["b1"], self.y1, self.n1, self.st1, s)
        f = self.n1[self.last]
        dl.disco_normalize_fwd(f, self.B, WIDTH, bf, self.u, bf, self.inv, s)
        dl.clip_loss_fwd_bwd(x["images"], self.u, self.B, WIDTH, S, bf, dl.DISCO_PATH_AUTO, self.loss, self.gI, self.gT, self.gs, ws, need, s)
        dl.disco_normalize_bwd(self.gT, f, bf, self.inv, self.B, WIDTH, self.df, s)
        self.dn1[self.last] = self.df.to(torch.bfloat16)
        small = self.small
        dl.disco_block_norm_bwd(self.s1, None, self.dn1, p, self.y1, x["gate"], None, None, x["w1"], self.st1, self.dy0, self.dp, small["gate"], None,
                                None, small["w1"], small["b1"], ws, need, s)
        do = (self.dp @ x["w_out"]).view(T, HEADS, HEAD)
        dq, dk, dv = (t.view(T, HEADS, HEAD) for t in self.dqkv.split(inner, 1))
        dl.disco_attention_bwd(self.sa, x["starts"], q, k, v, self.o, self.lse, do, dq, dk, dv, ws, need, s)
        dn0 = self.dqkv @ x["w_qkv"]
        dl.disco_block_norm_bwd(self.s0, self.dy0, dn0, None, self.y0, None, None, None, x["w0"], self.st0, self.dx, self.dh, None, None, None,
                                small["w0"], small["b0"], ws, need, s)
        grads = {"w_qkv": self.dqkv.T.float() @ self.n0.float(), "w_out": self.dp.T.float() @ self.o.view(T, inner).float(), "tokens": self.dh.clone(),
                 "places": self.dx.clone()} | {k: g.clone() for k, g in small.items()}
        taken = list(grads.values())
        dl.disco_grad_clip(taken, taken, self.max_norm, None, self.norm, ws, need, s)
        return grads


@pytest.mark.parametrize("B", [64, 96])
def test_a_step_of_a_text_tower(B):
    print("case tower step", B, flush=True)
    x = _inputs(B)
    loss, want, norm = _reference(x, None)
    step = Step(x, B, norm / 2)
    got = step.run()
    torch.cuda.synchronize()
    assert float(step.loss) == pytest.approx(loss, rel=1e-2)
    assert float(step.norm) == pytest.approx(norm, rel=BOUND)
    for name, g in got.items():
        # clipped to half of their norm
        off = float((g.double().cpu() * 2.0 - want[name]).norm() / want[name].norm())
        assert off <= BOUND + 2.0 ** -8, (name, off)


def test_the_step_twice_gives_equal_bits_on_another_stream():
    x = _inputs(64)
    step = Step(x, 64, 1e-3)
    one = {k: g.clone() for k, g in step.run().items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        two = step.run()
    side.synchronize()
    assert all(torch.equal(one[k], two[k]) for k in one)
