"""Attention: every invalid call is a status code before any GPU work."""
import pytest

import paper_2304_08480_amd as dl

FAKE = 0x1000


def _shape(**kw):
    a = dict(tokens=100, sequences=3, heads=8, kv_heads=2, head_dim=64, causal=1, dtype=dl.DISCO_BF16, scale=0.125, q_row=512, q_head=64,
             k_row=128, k_head=64, v_row=128, v_head=64, o_row=512, o_head=64)
    return dl.DiscoAttention(**(a | kw))


def _calls(shape, **kw):
    a = dict(starts=FAKE, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, n=1 << 30) | kw
    fwd = dl.disco_attention_fwd(shape, a["starts"], a["q"], a["k"], a["v"], a["o"], a["lse"], None, check=False) if "lse" in kw or \
        not set(kw) & {"dout", "dq", "dk", "dv", "ws", "n"} else None
    bwd = dl.disco_attention_bwd(shape, a["starts"], a["q"], a["k"], a["v"], a["o"], a["lse"], a["dout"], a["dq"], a["dk"], a["dv"], a["ws"], a["n"],
                                 None, check=False)
    return [s for s in (fwd, bwd) if s is not None]


@pytest.mark.parametrize("kw", [dict(tokens=0), dict(tokens=-1), dict(tokens=1 << 31), dict(sequences=0), dict(sequences=(1 << 24) + 1), dict(heads=0),
                                dict(kv_heads=0), dict(kv_heads=3), dict(heads=1 << 17), dict(head_dim=0), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(q_row=0), dict(k_head=-64), dict(o_row=(1 << 31) + 8),
                                dict(tokens=(1 << 31) - 1, heads=64, kv_heads=64)])
def test_bad_shapes(kw):
    assert set(_calls(_shape(**kw))) == {dl.DISCO_ERR_SHAPE}
    assert dl.disco_attention_workspace_bytes(_shape(**kw)) == 0


@pytest.mark.parametrize("kw", [dict(dtype=dl.DISCO_F32), dict(dtype=9), dict(head_dim=63), dict(head_dim=136), dict(q_row=516), dict(v_head=4)])
def test_unsupported(kw):
    assert set(_calls(_shape(**kw))) == {dl.DISCO_ERR_UNSUPPORTED}
    assert dl.disco_attention_workspace_bytes(_shape(**kw)) == 0


@pytest.mark.parametrize("name", ["starts", "q", "k", "v", "o", "lse", "dout", "dq", "dk", "dv"])
def test_null_and_misaligned_pointers(name):
    assert set(_calls(_shape(), **{name: None})) == {dl.DISCO_ERR_NULL}
    assert set(_calls(_shape(), **{name: FAKE + 2})) == {dl.DISCO_ERR_UNSUPPORTED}


def test_workspace():
    need = dl.disco_attention_workspace_bytes(_shape())
    assert need >= 100 * 8 * 4
    assert _calls(_shape(), ws=None) == [dl.DISCO_ERR_WORKSPACE]
    assert _calls(_shape(), ws=FAKE + 16) == [dl.DISCO_ERR_WORKSPACE]
    assert _calls(_shape(), n=need - 1) == [dl.DISCO_ERR_WORKSPACE]
    with pytest.raises(dl.DiscoError, match="disco_attention_fwd"):
        dl.disco_attention_fwd(_shape(heads=0), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE)


@pytest.mark.parametrize("kw", [dict(q_row=(1 << 22) + 8), dict(k_row=(1 << 22) + 8), dict(v_row=1 << 23), dict(o_row=1 << 24),
                                dict(sequences=1 << 20), dict(tokens=1 << 28, sequences=1), dict(sequences=8192, heads=1 << 10, kv_heads=1 << 10)])
def test_beyond_the_32_bits_of_a_tile_s_addresses_and_of_a_launch(kw):
    assert set(_calls(_shape(**kw))) == {dl.DISCO_ERR_SHAPE}
    assert dl.disco_attention_workspace_bytes(_shape(**kw)) == 0


def test_the_largest_row_stride_and_launch():
    assert dl.disco_attention_workspace_bytes(_shape(q_row=1 << 22, k_row=1 << 22, v_row=1 << 22, o_row=1 << 22)) > 0
    assert dl.disco_attention_workspace_bytes(_shape(sequences=(1 << 20) - 1)) > 0


def test_scales_past_fp32_in_base_2():
    # scores are taken times scale log2(e): 2.4e38 is fp32, its product is not, and 0 times that would be NaN
    assert set(_calls(_shape(scale=2.4e38))) == {dl.DISCO_ERR_SHAPE}
    assert dl.disco_attention_workspace_bytes(_shape(scale=2.4e38)) == 0
    assert dl.disco_attention_workspace_bytes(_shape(scale=2.3e38)) > 0
