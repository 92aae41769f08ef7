"""Block norm: every invalid call is a status code before any GPU work."""
import pytest

import paper_2304_08480_amd as dl

FAKE = 0x1000


def _shape(**kw):
    a = dict(rows=10, d=64, post=dl.DISCO_NORM_RMS, pre=dl.DISCO_NORM_LAYER, gate=dl.DISCO_GATE_CHANNEL, x_dtype=dl.DISCO_F32, h_dtype=dl.DISCO_BF16,
             eps_post=1e-5, eps_pre=1e-5, x_scale=1.0, h_scale=1.0)
    return dl.DiscoBlockNorm(**(a | kw))


def _fwd(shape=None, **kw):
    a = dict.fromkeys(("x", "h", "gate", "w_post", "b_post", "w_pre", "b_pre", "y", "n", "stats"), FAKE) | kw
    return dl.disco_block_norm_fwd(shape or _shape(), *a.values(), None, check=False)


def _bwd(shape=None, ws=FAKE, n=0, **kw):
    a = dict.fromkeys(("dy", "dn", "h", "y", "gate", "w_post", "b_post", "w_pre", "stats", "dx", "dh", "dgate", "dw_post", "db_post", "dw_pre", "db_pre"),
                      FAKE) | kw
    return dl.disco_block_norm_bwd(shape or _shape(), *a.values(), ws, n, None, check=False)


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=-1), dict(d=0), dict(d=8193), dict(rows=1 << 40), dict(eps_pre=-1e-5), dict(eps_post=float("nan")),
                                dict(x_scale=float("inf")), dict(h_scale=float("nan"))])
def test_bad_shapes(kw):
    assert _fwd(_shape(**kw)) == _bwd(_shape(**kw)) == dl.DISCO_ERR_SHAPE
    assert dl.disco_block_norm_workspace_bytes(_shape(**kw)) == 0


@pytest.mark.parametrize("kw", [dict(post=3), dict(pre=-1), dict(gate=3), dict(x_dtype=2), dict(h_dtype=-1)])
def test_unsupported(kw):
    assert _fwd(_shape(**kw)) == _bwd(_shape(**kw)) == dl.DISCO_ERR_UNSUPPORTED
    assert dl.disco_block_norm_workspace_bytes(_shape(**kw)) == 0


def test_pointers():
    for name in ("h", "gate", "y", "n", "stats"):
        assert _fwd(**{name: None}) == dl.DISCO_ERR_NULL, name
    for name in ("dn", "h", "y", "gate", "stats", "dh"):
        assert _bwd(**{name: None}) == dl.DISCO_ERR_NULL, name
    assert _bwd(_shape(pre=dl.DISCO_NORM_NONE), dy=None) == dl.DISCO_ERR_NULL
    for name in ("x", "y", "stats", "w_post", "b_pre", "gate"):
        assert _fwd(**{name: FAKE + 2}) == dl.DISCO_ERR_UNSUPPORTED, name
    assert _fwd(h=FAKE + 1) == _bwd(dn=FAKE + 1) == _bwd(dw_pre=FAKE + 2) == _bwd(dgate=FAKE + 2) == dl.DISCO_ERR_UNSUPPORTED
    need = dl.disco_block_norm_workspace_bytes(_shape())
    assert need > 0
    assert _bwd(n=need - 1) == _bwd(ws=None, n=need) == _bwd(ws=FAKE + 16, n=need) == dl.DISCO_ERR_WORKSPACE
    with pytest.raises(dl.DiscoError, match="disco_block_norm_bwd"):
        dl.disco_block_norm_bwd(_shape(), *([None] * 17), 0)
