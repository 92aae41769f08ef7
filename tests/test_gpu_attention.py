"""disco_attention_fwd and disco_attention_bwd against the float64 oracle, every entry within the bound that the oracle derives for it."""
import pytest
import torch

import paper_2304_08480_amd as dl
from oracle import attention as oa

pytestmark = pytest.mark.gpu


class Attention:
    """Buffers of one packed batch: a fused projection output, or separate tensors with room between rows and heads."""

    def __init__(self, lengths, heads, kv_heads, dim, causal, seed=0, first=0, behind=0, fused=True, scale=None, gap=0, sharp=1.0):
        g = torch.Generator().manual_seed(seed)
        starts = [first]
        for n in lengths:
            starts.append(starts[-1] + n)
        T = starts[-1] + behind
        self.T, self.H, self.G, self.D, self.causal, self.starts_host = T, heads, kv_heads, dim, causal, starts
        self.scale = dim ** -0.5 if scale is None else scale

        def make(n, spread=1.0):
            return (torch.randn(T, n, dim, generator=g) * spread).to(torch.bfloat16)

        self.host = [make(heads, sharp), make(kv_heads), make(kv_heads), make(heads)]
        self.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        row = {"q": heads, "k": kv_heads, "v": kv_heads, "o": heads}
        if fused:
            buffer = torch.cat(self.host[:3], 1).cuda()
            grads = torch.full_like(buffer, float("nan"))
            cut = (heads, kv_heads, kv_heads)
            self.q, self.k, self.v = buffer.split(cut, 1)
            self.dq, self.dk, self.dv = grads.split(cut, 1)
            self.do = self.host[3].cuda()
            self.o = torch.full_like(self.do, float("nan"))
        else:
            def place(t, n):
                wide = torch.full((T, n + 1, dim + gap), float("nan"), dtype=torch.bfloat16, device="cuda")
                view = wide[:, :n, :dim]
                if t is not None:
                    view.copy_(t)
                return view

            self.q, self.k, self.v, self.do = (place(t, t.shape[1]) for t in self.host)
            self.o, self.dq, self.dk, self.dv = (place(None, n) for n in (heads, heads, kv_heads, kv_heads))
        self.lse = torch.full((heads, T), float("nan"), device="cuda")
        strides = {m + "_" + way: getattr(self, m).stride(i) for m in row for i, way in enumerate(("row", "head"))}
        self.shape = dl.DiscoAttention(tokens=T, sequences=len(lengths), heads=heads, kv_heads=kv_heads, head_dim=dim, causal=int(causal),
                                       dtype=dl.DISCO_BF16, scale=self.scale, **strides)
        self.need = dl.disco_attention_workspace_bytes(self.shape)
        self.ws = torch.full((self.need,), 255, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None):
        dl.disco_attention_fwd(self.shape, self.starts, self.q, self.k, self.v, self.o, self.lse, stream or torch.cuda.current_stream())

    def backward(self, stream=None):
        dl.disco_attention_bwd(self.shape, self.starts, self.q, self.k, self.v, self.o, self.lse, self.do, self.dq, self.dk, self.dv, self.ws,
                               self.need, stream or torch.cuda.current_stream())

    def outputs(self):
        return {n: getattr(self, n).float().cpu() for n in ("o", "lse", "dq", "dk", "dv")}

    def check(self):
        want = oa.packed(*(t.double() for t in self.host[:3]), self.starts_host, self.scale, self.causal, self.host[3].double())
        for name, got in self.outputs().items():
            value, bound = want[name]
            outside = torch.isinf(bound)
            assert torch.isnan(got[outside]).all(), name + ": rows of no sequence were written"
            off = (got.double() - value).abs()[~outside] / bound[~outside].clamp(min=1e-30)
            assert not off.numel() or float(off.max()) <= 1.0, (name, float(off.max()))


LENGTHS = [[1], [2, 1], [31], [32], [33], [64, 0, 65], [127, 128, 129], [5, 0, 0, 77, 1, 30], [300, 1, 200]]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("dim", [64, 128])
def test_lengths(lengths, dim, causal):
    print("case attention", lengths, dim, causal, flush=True)
    a = Attention(lengths, 4, 2, dim, causal, seed=len(lengths))
    a.forward()
    a.backward()
    a.check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 72, 80, 96, 104, 120])
@pytest.mark.parametrize("lengths", [[3, 40, 9], [70, 140]], ids=str)
def test_head_widths(lengths, dim, causal):
    print("case attention width", lengths, dim, causal, flush=True)
    a = Attention(lengths, 3, 3, dim, causal, seed=dim)
    a.forward()
    a.backward()
    a.check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 1), (6, 2), (8, 8), (12, 3)])
def test_shared_heads_strides_and_rows_of_no_sequence(heads, kv_heads):
    print("case attention heads", heads, kv_heads, flush=True)
    for lengths in ([17, 33, 64], [200, 111]):
        a = Attention(lengths, heads, kv_heads, 64, True, seed=heads, first=5, behind=9, fused=False, gap=8)
        a.forward()
        a.backward()
        a.check()


@pytest.mark.parametrize("scale,sharp", [(1e-3, 1.0), (0.125, 12.0), (2.0, 3.0)])
def test_flat_and_saturated_softmax(scale, sharp):
    a = Attention([90, 150], 2, 2, 64, True, scale=scale, sharp=sharp)
    a.forward()
    a.backward()
    a.check()


def test_thousands_of_short_sequences():
    g = torch.Generator().manual_seed(3)
    lengths = torch.randint(0, 9, (5000,), generator=g).tolist()
    a = Attention(lengths, 2, 1, 32, True)
    a.forward()
    a.backward()
    a.check()


def test_equal_calls_give_equal_bits_and_neighbours_do_not_matter():
    a = Attention([50, 0, 300, 77], 4, 2, 64, True)
    a.forward()
    a.backward()
    one = a.outputs()
    a.forward()
    a.backward()
    assert all(torch.equal(one[n], x) for n, x in a.outputs().items())
    # what is not finite stays within its sequence
    for t in (a.q, a.k, a.v, a.do):
        t[50:60] = float("nan")
        t[345:350] = float("inf")
    a.forward()
    a.backward()
    for n, x in a.outputs().items():
        y = one[n]
        if n == "lse":
            x, y = x.T, y.T
        assert torch.equal(x[:50], y[:50]) and torch.equal(x[350:], y[350:]), n
        assert torch.isnan(x[50:350]).any()


def test_captured_and_on_another_stream():
    a, b = (Attention([40, 90, 3], 4, 2, 64, True, seed=s) for s in (1, 2))
    eager = []
    for x in (a, b):
        x.forward()
        x.backward()
        eager.append(x.outputs())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in (a, b):
            x.forward()
            x.backward()
    for _ in range(3):
        for x in (a, b):
            for t in (x.o, x.lse, x.dq, x.dk, x.dv):
                t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for x, want in zip((a, b), eager):
            assert all(torch.equal(want[n], y) for n, y in x.outputs().items())
    # two calls at once
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for x, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            x.forward(s)
            x.backward(s)
    torch.cuda.synchronize()
    for x, want in zip((a, b), eager):
        assert all(torch.equal(want[n], y) for n, y in x.outputs().items())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [32, 64, 88, 128])
@pytest.mark.parametrize("typical,longer", [(18, 33), (18, 300), (30, 97), (40, 700), (100, 129), (180, 257), (190, 500)])
def test_many_short_sequences_and_a_few_longer_ones(typical, longer, dim, causal):
    # sequences of every length around the typical one, in a batch whose mean says short; the longer ones first, amid and last
    print("case attention mixed", typical, longer, dim, causal, flush=True)
    g = torch.Generator().manual_seed(typical)
    n = 70 if typical < 100 else 24
    lengths = torch.randint(max(0, typical // 3), typical + typical // 3 + 1, (n,), generator=g).tolist()
    lengths = [longer] + lengths[:n // 2] + [longer, 0] + lengths[n // 2:] + [longer + 1]
    a = Attention(lengths, 2, 2, dim, causal, seed=dim, behind=3)
    a.forward()
    a.backward()
    a.check()


@pytest.mark.parametrize("kv_heads", [1, 2])
def test_short_sequences_on_both_sides_of_their_limit(kv_heads):
    for n in (8192, 8193):
        g = torch.Generator().manual_seed(n)
        a = Attention(torch.randint(0, 5, (n,), generator=g).tolist(), 2, kv_heads, 32, True, seed=n)
        a.forward()
        a.backward()
        a.check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (3, 1, 128), (4, 2, 32), (8, 2, 96), (20, 2, 64), (20, 20, 64), (20, 20, 128)])
def test_long_sequences_on_few_and_many_heads(heads, kv_heads, dim, causal):
    print("case attention long", heads, kv_heads, dim, causal, flush=True)
    a = Attention([1100, 3, 900, 97], heads, kv_heads, dim, causal, seed=heads)
    a.forward()
    a.backward()
    a.check()
    one = a.outputs()
    a.forward()
    a.backward()
    assert all(torch.equal(one[n], x) for n, x in a.outputs().items())


def test_the_largest_row_stride_with_tiles_of_many_rows():
    # 700 rows, 8 MiB apart: the rows of a walked tile span 2 GiB
    print("case attention largest row stride", flush=True)
    a = Attention([650, 50], 2, 1, 64, True, seed=9, scale=0.3)
    a.forward()
    a.backward()
    want = a.outputs()
    room, grads = (torch.empty(700, 1 << 22, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for j, n in enumerate("qkvo"):
        wide = [t[:, 1024 * j:1024 * j + getattr(a, n).shape[1] * 64].view(700, -1, 64) for t in (room, grads)]
        if n == "o":
            a.o = wide[0]
            do = grads[:, 1 << 21:(1 << 21) + 128].view(700, 2, 64)
            do.copy_(a.do)
            a.do = do
        else:
            wide[0].copy_(getattr(a, n))
            setattr(a, n, wide[0])
            setattr(a, "d" + n, wide[1])
        setattr(a.shape, n + "_row", 1 << 22)
        setattr(a.shape, n + "_head", 64)
    a.forward()
    a.backward()
    got = a.outputs()
    assert all(torch.equal(got[k], want[k]) for k in got)


@pytest.mark.parametrize("lengths,heads", [([300], 2), ([200, 200], 40), ([96] * 80, 2), ([30] * 300, 2)], ids=str)
def test_how_far_a_masked_nan_reaches(lengths, heads):
    # the last row of the last sequence: no other sequence sees it, nor a row more than 63 ahead of it, in any direction of the pass
    a = Attention(lengths, heads, heads, 64, True, seed=5)
    a.forward()
    a.backward()
    want = a.outputs()
    for t in (a.q, a.k, a.v, a.do):
        t[-1] = float("nan")
    a.forward()
    assert torch.equal(a.o[:a.T - 64].float().cpu(), want["o"][:a.T - 64])
    assert torch.equal(a.lse[:, :a.T - 1].cpu(), want["lse"][:, :a.T - 1])
    a.backward()
    got = a.outputs()
    first = a.T - lengths[-1]
    for n in ("dq", "dk", "dv"):
        assert torch.equal(got[n][:first], want[n][:first]), n
    assert torch.equal(got["dq"][:a.T - 64], want["dq"][:a.T - 64])
    assert torch.isnan(got["dk"][a.T - 1]).all() and torch.isnan(got["o"][a.T - 1]).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [32, 64])
@pytest.mark.parametrize("typical,longer", [(18, 64), (18, 65), (30, 97), (40, 128), (40, 300), (60, 193), (62, 257)])
def test_thousands_of_short_sequences_and_heads(typical, longer, dim, causal):
    # as above, where there are more than a few of them
    print("case attention many", typical, longer, dim, causal, flush=True)
    g = torch.Generator().manual_seed(typical + longer)
    lengths = torch.randint(0, 2 * typical + 1, (330,), generator=g).tolist()
    a = Attention([longer] + lengths[:160] + [longer, 0, 32, 33] + lengths[160:] + [longer + 1], 4, 4, dim, causal, seed=dim, behind=3)
    a.forward()
    a.backward()
    a.check()


@pytest.mark.parametrize("heads,kv_heads,dim,causal,lengths", [(8, 8, 64, False, [695, 1063, 2000]), (8, 4, 128, True, [100, 923, 0, 2000, 1083, 1683]),
                                                               (6, 2, 96, True, [1500, 31, 1601, 1]), (8, 8, 64, True, [2845, 1, 710, 128, 129])])
def test_tiles_with_two_sets_of_waves(heads, kv_heads, dim, causal, lengths):
    print("case attention two sets", heads, kv_heads, dim, causal, lengths, flush=True)
    a = Attention(lengths, heads, kv_heads, dim, causal, seed=dim, behind=5)
    a.forward()
    a.backward()
    a.check()
