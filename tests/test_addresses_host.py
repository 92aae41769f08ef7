"""What the binding takes for a device address: an int, also one of a class of its own, and anything with a data_ptr()."""
import enum

import pytest
import torch

import paper_2304_08480_amd as dl
from paper_2304_08480_amd import binding


class Address(int):
    """An address with a note on it."""


class Buffers(enum.IntEnum):
    FEATURES = 0x1000


@pytest.mark.parametrize("at", [0x1000, Address(0x1000), Buffers.FEATURES], ids=lambda a: type(a).__name__)
def test_addresses(at):
    assert binding._ptr(at) == 0x1000
    shape = dl.DiscoAttention()                                  # all zeros: refused, after the arguments were taken
    assert dl.disco_attention_fwd(shape, *[at] * 6, check=False) == dl.DISCO_ERR_SHAPE
    assert dl.disco_loss_fwd_bwd(at, at, 0, 8, 0, 1, 1.0, dl.DISCO_F32, dl.DISCO_PATH_AUTO, 0, at, at, at, at, at, 0, None,
                                 check=False) == dl.DISCO_ERR_SHAPE


def test_tensors_and_nothing():
    t = torch.zeros(4)
    assert binding._ptr(t) == t.data_ptr() and binding._ptr(None) is None
    with pytest.raises(AttributeError):
        binding._ptr(1.5)
