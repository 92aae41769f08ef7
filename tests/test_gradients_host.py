"""Gradient norm and clipping: every invalid call is a status code before any GPU work; lists are read on the host."""
import ctypes

import pytest
import torch

import paper_2304_08480_amd as dl
from paper_2304_08480_amd import binding

FAKE = 0x1000


def _list(n=2, **kw):
    a = dict(src=[FAKE] * n, dst=[FAKE] * n, elements=[100] * n, dtypes=[dl.DISCO_F32] * n) | kw
    return ((ctypes.c_void_p * n)(*a["src"]), (ctypes.c_void_p * n)(*a["dst"]), (ctypes.c_int64 * n)(*a["elements"]), (ctypes.c_int32 * n)(*a["dtypes"]))


def _calls(lists, count=2, norm=FAKE, ws=FAKE, n=1 << 30, max_norm=1.0):
    src, dst, elements, dtypes = lists
    return {binding._lib.disco_grad_norm(src, elements, dtypes, count, 0, norm, ws, n, None),
            binding._lib.disco_grad_clip(src, dst, elements, dtypes, count, max_norm, None, norm, ws, n, None)}


def test_refusals():
    ok = _list()
    assert _calls(ok, norm=None) == {dl.DISCO_ERR_NULL}
    assert _calls(_list(src=[FAKE, None])) == {dl.DISCO_ERR_NULL}
    assert _calls((None, None, ok[2], ok[3])) == {dl.DISCO_ERR_NULL}
    assert _calls((ok[0], ok[1], None, ok[3])) == {dl.DISCO_ERR_NULL}
    assert _calls(_list(elements=[1, -1])) == {dl.DISCO_ERR_SHAPE}
    assert _calls(_list(elements=[1, (1 << 40) + 1])) == {dl.DISCO_ERR_SHAPE}
    assert _calls(ok, count=-1) == _calls(ok, count=(1 << 20) + 1) == {dl.DISCO_ERR_SHAPE}
    assert _calls(_list(20, elements=[1 << 40] * 20), count=20) == {dl.DISCO_ERR_SHAPE}
    assert _calls(_list(dtypes=[0, 2])) == {dl.DISCO_ERR_UNSUPPORTED}
    assert _calls(_list(src=[FAKE, FAKE + 2])) == {dl.DISCO_ERR_UNSUPPORTED}
    assert _calls(ok, norm=FAKE + 2) == {dl.DISCO_ERR_UNSUPPORTED}
    need = dl.disco_grad_workspace_bytes(2)
    assert _calls(ok, ws=None) == _calls(ok, ws=FAKE + 8) == _calls(ok, n=need - 1) == {dl.DISCO_ERR_WORKSPACE}
    for bad in (0.0, -1.0, float("nan")):
        assert dl.DISCO_ERR_SHAPE in _calls(ok, n=need - 1, max_norm=bad)
    src, _, elements, dtypes = ok
    assert binding._lib.disco_grad_clip(src, None, elements, dtypes, 2, 1.0, None, FAKE, FAKE, need, None) == dl.DISCO_ERR_NULL


def test_workspace_grows_with_the_list():
    assert dl.disco_grad_workspace_bytes(-1) == dl.disco_grad_workspace_bytes((1 << 20) + 1) == 0
    assert 0 < dl.disco_grad_workspace_bytes(0) <= dl.disco_grad_workspace_bytes(100) < dl.disco_grad_workspace_bytes(1000)


def test_lists_of_tensors():
    a, b = torch.zeros(4, 6), torch.zeros(5, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):
        dl.disco_grad_norm([a.T], FAKE, FAKE, 1 << 20)
    with pytest.raises(ValueError, match="sizes or types"):
        dl.disco_grad_clip([a, b], [b, a], 1.0, None, FAKE, FAKE, 1 << 20)
    assert dl.disco_grad_norm([a.half()], FAKE, FAKE, 1 << 20, check=False) == dl.DISCO_ERR_UNSUPPORTED
    with pytest.raises(dl.DiscoError, match="disco_grad_clip"):
        dl.disco_grad_clip([a.half()], [a.half()], 1.0, None, FAKE, FAKE, 1 << 20)


def test_more_pieces_than_a_workgroup_counts():
    # pieces of 8192 elements: 2^31 - 1 - 1000 of them, and past them the step of 2048 workgroups
    rest = ((1 << 31) - 1 - 1000 - 15 * ((1 << 27) + 1) - 1) * 8192
    assert rest < 1 << 40
    assert _calls(_list(16, elements=[1 << 40] * 15 + [rest]), count=16) == {dl.DISCO_ERR_SHAPE}
