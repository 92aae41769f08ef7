"""disco_block_norm_fwd and disco_block_norm_bwd against the float64 oracle.

Tolerances.  STEP is half a step of the stored type relative to a value (bf16 2^-8, fp32 2^-24).  Everything before a store is fp32: at most d
additions in trees and about 20 operations, each 2^-24 of the largest intermediate.  The sums of a row run 8 deep in a lane and at most 10 over
lanes, 18 roundings; 64 of 2^-24 cover them, the statistics and the rest.  The entry's scale is what its formula adds up: for n it is
(|z| + mean|z|) rstd |w| + |b|, for gradients the row's rstd (|a| + mean|a| + |zhat| mean|a zhat|), |zhat| taken as (|z| + mean|z|) rstd.
It is mean|z| and not |mean|: d roundings of a sum of terms z / d, s deep, leave s 2^-24 sum |z| / d in the mean, however small the mean comes out (a
row that was normed once already has a mean of about 0 and entries of about 0, whose difference carries that error)."""
import pytest
import torch

import paper_2304_08480_amd as dl
from oracle import block_norm as ob

pytestmark = pytest.mark.gpu
KINDS = {"none": dl.DISCO_NORM_NONE, "layer": dl.DISCO_NORM_LAYER, "rms": dl.DISCO_NORM_RMS}
GATES = {"none": dl.DISCO_GATE_NONE, "channel": dl.DISCO_GATE_CHANNEL, "element": dl.DISCO_GATE_ELEMENT}
TYPES = {"bf16": (dl.DISCO_BF16, torch.bfloat16, 2.0 ** -8), "f32": (dl.DISCO_F32, torch.float32, 2.0 ** -24)}
FP32 = 64 * 2.0 ** -24
EPS = 1e-5


class Norm:
    def __init__(self, rows, d, post="none", pre="layer", gate="none", x="bf16", h="bf16", seed=0, with_x=True, shift=0.0, bias=True, weight=True):
        g = torch.Generator().manual_seed(seed)

        def r(*shape, t="f32", scale=1.0, add=0.0):
            return (torch.randn(*shape, generator=g) * scale + add).to(TYPES[t][1])

        self.rows, self.d, self.post, self.pre, self.gate_kind, self.xt, self.ht = rows, d, post, pre, gate, x, h
        host = {"x": r(rows, d, t=x, scale=2.0, add=shift) if with_x else None, "h": r(rows, d, t=h, add=shift),
                "gate": {"none": None, "channel": r(d), "element": r(rows, d, t=h)}[gate],
                "dy": r(rows, d, t=x, scale=0.1), "dn": r(rows, d, t=h, scale=0.1) if pre != "none" else None}
        for k, kind in (("post", post), ("pre", pre)):
            host["w_" + k] = 1.0 + 0.3 * r(d) if weight and kind != "none" else None
            host["b_" + k] = 0.2 * r(d) if bias and kind == "layer" else None
        self.host = host
        self.dev = {k: None if v is None else v.cuda() for k, v in host.items()}
        nan = float("nan")
        for name, t in (("y", x), ("n", h), ("dx", x), ("dh", h)):
            self.dev[name] = torch.full((rows, d), nan, dtype=TYPES[t][1], device="cuda")
        self.dev["dgate"] = None if gate == "none" else torch.full_like(self.dev["gate"], nan)
        for k in ("w_post", "b_post", "w_pre", "b_pre"):
            self.dev["d" + k] = None if host[k] is None else torch.full((d,), nan, device="cuda")
        self.dev["stats"] = torch.full((rows, 4), nan, device="cuda")
        self.x_scale, self.h_scale = 0.875, 0.75
        self.shape = dl.DiscoBlockNorm(rows=rows, d=d, post=KINDS[post], pre=KINDS[pre], gate=GATES[gate], x_dtype=TYPES[x][0], h_dtype=TYPES[h][0],
                                       eps_post=EPS, eps_pre=EPS, x_scale=self.x_scale, h_scale=self.h_scale)
        self.need = dl.disco_block_norm_workspace_bytes(self.shape)
        self.ws = torch.full((self.need,), 255, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None):
        v = self.dev
        dl.disco_block_norm_fwd(self.shape, v["x"], v["h"], v["gate"], v["w_post"], v["b_post"], v["w_pre"], v["b_pre"], v["y"],
                                v["n"] if self.pre != "none" else None, v["stats"], stream or torch.cuda.current_stream())

    def backward(self, stream=None):
        v = self.dev
        dl.disco_block_norm_bwd(self.shape, v["dy"], v["dn"], v["h"], v["y"], v["gate"], v["w_post"], v["b_post"], v["w_pre"], v["stats"], v["dx"],
                                v["dh"], v["dgate"], v["dw_post"], v["db_post"], v["dw_pre"], v["db_pre"], self.ws, self.need,
                                stream or torch.cuda.current_stream())

    OUTPUTS = ("y", "n", "stats", "dx", "dh", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")

    def outputs(self):
        return {k: self.dev[k].float().cpu() for k in self.OUTPUTS if self.dev[k] is not None and (k != "n" or self.pre != "none")}

    def check(self):
        got = self.outputs()
        w = {k: None if v is None else v.double() for k, v in self.host.items()}
        xs, hs = TYPES[self.xt][2], TYPES[self.ht][2]
        ystored = got["y"].double()
        y, _, _ = ob.forward(w["x"], w["h"], w["gate"], self.post, self.pre, EPS, self.x_scale, self.h_scale, w["w_post"], w["b_post"], w["w_pre"],
                             w["b_pre"])

        def parts(z, kind, weight, b):
            """What N adds up, in absolute values."""
            _, rstd = ob.statistics(z, kind, EPS)
            return ((z.abs() + z.abs().mean(1, keepdim=True)) * rstd * (1.0 if weight is None else weight.abs())) + (0.0 if b is None else b.abs())

        def near(name, value, bound):
            off = (got[name].double() - value).abs() - bound
            assert float(off.max()) <= 0.0, (name, float(off.max()), float(value.abs().max()))

        up = parts(w["h"], self.post, w["w_post"], w["b_post"]) if self.post != "none" else w["h"].abs()
        yp = self.h_scale * up * (1.0 if w["gate"] is None else w["gate"].abs()) + (0.0 if w["x"] is None else self.x_scale * w["x"].abs())
        near("y", y, xs * y.abs() + FP32 * yp + 1e-38)
        if self.pre != "none":
            n = ob.norm(ystored, self.pre, EPS, w["w_pre"], w["b_pre"])
            near("n", n, hs * n.abs() + FP32 * parts(ystored, self.pre, w["w_pre"], w["b_pre"]))
        # the variance of a row of mean m and deviation s carries what the rounding of its mean and of its deviations from it leaves: 2^-24 |m| / s
        for at, z, kind in ((0, w["h"], self.post), (2, ystored, self.pre)):
            mean, rstd = ob.statistics(z, kind, EPS)
            m, r = got["stats"][:, at:at + 1].double(), got["stats"][:, at + 1:at + 2].double()
            assert float(((m - mean).abs() - FP32 * z.abs().mean(1, keepdim=True)).max()) <= 0
            assert float(((r - rstd).abs() - FP32 * rstd * (1 + z.abs().amax(1, keepdim=True) * rstd)).max()) <= 0
        want = ob.backward(w["dy"], w["dn"], w["h"], ystored, w["gate"], self.post, self.pre, EPS, self.x_scale, self.h_scale, w["w_post"], w["b_post"],
                           w["w_pre"])

        def spread(g, z, kind, weight):
            """What N' adds up, and the error of zhat in each."""
            _, rstd = ob.statistics(z, kind, EPS)
            zh = (z.abs() + z.abs().mean(1, keepdim=True)) * rstd
            a = g.abs() if weight is None else g.abs() * weight.abs()
            return rstd * (a + a.mean(1, keepdim=True) + 3 * zh * (a * zh).mean(1, keepdim=True)), (g.abs() * zh).sum(0), g.abs().sum(0)

        t_off = FP32 * w["dy"].abs()
        if self.pre != "none":
            s, sw, sb = spread(w["dn"], ystored, self.pre, w["w_pre"])
            t_off = t_off + FP32 * s
            for k, v in (("dw_pre", sw), ("db_pre", sb)):
                if k in got:
                    near(k, want[k], FP32 * v)
        t = want["dx"] / self.x_scale
        near("dx", want["dx"], xs * want["dx"].abs() + self.x_scale * (t_off + FP32 * t.abs()) + 1e-38)
        g = 1.0 if w["gate"] is None else w["gate"].abs()
        t_all = t_off + FP32 * t.abs()
        if self.gate_kind == "element":
            near("dgate", want["dgate"], hs * want["dgate"].abs() + self.h_scale * (t_all * up + FP32 * t.abs() * up))
        if self.gate_kind == "channel":
            near("dgate", want["dgate"].sum(0), self.h_scale * (t_all * up + FP32 * t.abs() * up).sum(0))
        du, du_off = self.h_scale * g * t.abs(), self.h_scale * g * t_all
        if self.post == "none":
            near("dh", want["dh"], hs * want["dh"].abs() + du_off + FP32 * du + 1e-38)
        else:
            s, sw, sb = spread(du, w["h"], self.post, w["w_post"])
            o, ow, ob_ = spread(du_off, w["h"], self.post, w["w_post"])
            near("dh", want["dh"], hs * want["dh"].abs() + FP32 * s + o)
            for k, v in (("dw_post", FP32 * sw + ow), ("db_post", FP32 * sb + ob_)):
                if k in got:
                    near(k, want[k], v)


@pytest.mark.parametrize("d", [1, 7, 8, 64, 77, 128, 129, 255, 512, 520, 768, 1001, 2048, 2049, 4096, 5000, 8191, 8192])
@pytest.mark.parametrize("rows", [1, 3, 37])
def test_widths(rows, d):
    print("case block norm", rows, d, flush=True)
    n = Norm(rows, d, post="layer", pre="layer", gate="channel", x="f32", seed=d)
    n.forward()
    n.backward()
    n.check()


@pytest.mark.parametrize("gate", ["none", "channel", "element"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
def test_forms(post, pre, gate):
    for x, h, d in (("bf16", "bf16", 320), ("f32", "bf16", 77), ("bf16", "f32", 1500), ("f32", "f32", 33)):
        print("case block norm", post, pre, gate, x, h, d, flush=True)
        n = Norm(29, d, post, pre, gate, x, h, seed=d)
        n.forward()
        n.backward()
        n.check()


def test_many_rows():
    for d in (40, 512):
        n = Norm(20011, d, "rms", "layer", "channel", "bf16", "bf16")
        n.forward()
        n.backward()
        n.check()


def test_absent_parts():
    n = Norm(50, 96, "layer", "layer", "none", "f32", "f32", with_x=False, bias=False, weight=False)
    n.forward()
    n.backward()
    n.check()
    # gradients that are not wanted, and no gradient from the stream
    full = n.outputs()
    v = n.dev
    v["dh"].fill_(0)
    dl.disco_block_norm_bwd(n.shape, v["dy"], v["dn"], v["h"], v["y"], None, None, None, None, v["stats"], None, v["dh"], None, None, None, None, None,
                            n.ws, n.need, torch.cuda.current_stream())
    assert torch.equal(v["dh"].float().cpu(), full["dh"])
    v["dy"].zero_()
    n.backward()
    zero = n.outputs()
    dl.disco_block_norm_bwd(n.shape, None, v["dn"], v["h"], None if n.pre == "none" else v["y"], None, None, None, None, v["stats"], v["dx"], v["dh"],
                            None, None, None, None, None, n.ws, n.need, torch.cuda.current_stream())
    assert torch.equal(v["dx"].float().cpu(), zero["dx"]) and torch.equal(v["dh"].float().cpu(), zero["dh"])


def test_a_mean_far_from_zero_and_constant_rows():
    n = Norm(20, 256, "layer", "layer", "none", "f32", "f32", shift=100.0)
    n.dev["h"][3] = 5.0
    n.host["h"][3] = 5.0
    n.dev["x"][3] = 2.0
    n.host["x"][3] = 2.0
    n.forward()
    assert torch.isfinite(n.dev["n"]).all()
    n.backward()
    n.check()


@pytest.mark.parametrize("x,h", [("bf16", "bf16"), ("f32", "f32")])
def test_in_place_unaligned_and_not_finite(x, h):
    n = Norm(41, 131, "rms", "layer", "element", x, h)
    n.forward()
    n.backward()
    want = n.outputs()
    v, d = n.dev, n.d
    # rows that start at any element: y over x, n over h, dx over dy, dh over dn
    places = {}
    for k in ("x", "h", "gate", "dy", "dn"):
        room = torch.zeros(v[k].numel() + 3, dtype=v[k].dtype, device="cuda")
        places[k] = room[3:].view_as(v[k])
        places[k].copy_(v[k])
    h0 = v["h"].clone()
    dl.disco_block_norm_fwd(n.shape, places["x"], places["h"], places["gate"], v["w_post"], v["b_post"], v["w_pre"], v["b_pre"], places["x"], places["h"],
                            v["stats"], torch.cuda.current_stream())
    assert torch.equal(places["x"].float().cpu(), want["y"]) and torch.equal(places["h"].float().cpu(), want["n"])
    dl.disco_block_norm_bwd(n.shape, places["dy"], places["dn"], h0, places["x"], places["gate"], v["w_post"], v["b_post"], v["w_pre"], v["stats"],
                            places["dy"], places["dn"], v["dgate"], v["dw_post"], v["db_post"], v["dw_pre"], v["db_pre"], n.ws, n.need,
                            torch.cuda.current_stream())
    assert torch.equal(places["dy"].float().cpu(), want["dx"]) and torch.equal(places["dn"].float().cpu(), want["dh"])
    # one row that is not finite: the others keep their values
    v["h"][7, 5] = float("nan")
    v["x"][40, 0] = float("inf")
    n.forward()
    n.backward()
    got = n.outputs()
    rest = [i for i in range(41) if i not in (7, 40)]
    for k in ("y", "n", "dx", "dh", "dgate"):
        assert torch.equal(got[k][rest], want[k][rest]), k
    assert torch.isnan(got["y"][7]).any() and torch.isnan(got["dw_post"]).any()


def test_captured_twice_and_on_two_streams():
    a, b = Norm(300, 512, "layer", "rms", "channel", seed=1), Norm(3000, 200, "none", "layer", "channel", seed=2)
    eager = []
    for n in (a, b):
        n.forward()
        n.backward()
        eager.append(n.outputs())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for n in (a, b):
            n.forward()
            n.backward()
    for _ in range(3):
        for n in (a, b):
            for k in n.outputs():
                n.dev[k].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for n, want in zip((a, b), eager):
            assert all(torch.equal(want[k], x) for k, x in n.outputs().items())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for n, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            n.forward(s)
            n.backward(s)
    torch.cuda.synchronize()
    for n, want in zip((a, b), eager):
        assert all(torch.equal(want[k], x) for k, x in n.outputs().items())


@pytest.mark.parametrize("rows,d", [(17, 100), (5, 500), (2049, 130)])
def test_an_infinity_in_the_last_row_of_a_workgroup_that_has_rows_to_spare(rows, d):
    """A workgroup's places behind the last row add nothing to the sums, whatever the last row holds: sums of one infinity are infinite, not NaN."""
    n = Norm(rows, d, "layer", "none", "channel", "f32", "f32")
    n.forward()
    n.dev["dy"][rows - 1] = 1e30
    n.shape.x_scale = 1e30                                      # dx = x_scale dy is infinite
    n.backward()
    want = n.outputs()
    assert torch.isinf(want["dx"][rows - 1]).all() and all(torch.isfinite(want[k]).all() for k in ("dgate", "dw_post", "db_post"))
    v = n.dev
    dl.disco_block_norm_bwd(n.shape, v["dy"], v["dn"], v["h"], v["y"], v["gate"], v["w_post"], v["b_post"], v["w_pre"], v["stats"], v["dy"], v["dh"],
                            v["dgate"], v["dw_post"], v["db_post"], v["dw_pre"], v["db_pre"], n.ws, n.need, torch.cuda.current_stream())
    v["dx"] = v["dy"]
    got = n.outputs()
    assert all(torch.equal(got[k], want[k]) for k in got)
    n = Norm(rows, d, "none", "layer", "none", "f32", "f32")
    n.forward()
    n.dev["dn"][rows - 1, 3] = float("inf")
    n.backward()
    got = n.outputs()
    assert got["db_pre"][3] == float("inf") and torch.isfinite(got["db_pre"][[i for i in range(d) if i != 3]]).all()
    assert torch.equal(torch.isnan(got["dw_pre"]), torch.zeros(d, dtype=torch.bool))
