"""Products of more tiles than a launch holds (2^32 lanes): HEDDLE_E_RANGE from
the host. The addresses are of no memory; nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_2609_34244_amd import heddle as H

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would run on no memory")

X, W, Y, ROWS = 1 << 44, 1 << 45, 1 << 46, 1 << 30


def linear(**over):
    d = dict(dtype=H.HEDDLE_T_BF16, act=H.HEDDLE_A_NONE, m=ROWS, n=256, k=8, x=X, ldx=8, w=W, ldw=8, y=Y, ldy=256)
    d.update(over)
    return H.heddle_linear_desc(**d)


@pytest.mark.parametrize("n", [256, 1024, 1 << 16, 1 << 22])
def test_too_many_tiles(n):
    d = linear(n=n, ldy=n)
    assert H.lib().heddle_linear(C.byref(d), None, 0, None) == H.HEDDLE_E_RANGE, H.heddle_last_error()


def test_too_many_tiles_of_groups():
    d = linear(n=256, d_offsets=1 << 20, groups=65535, stride_w=256 * 8)
    assert H.lib().heddle_linear(C.byref(d), None, 0, None) == H.HEDDLE_E_RANGE, H.heddle_last_error()


def test_fewer_are_launched():
    """2^23 tiles of 128 x 128, 2^31 lanes: ends for want of a GPU"""
    d = linear(n=64, ldy=64)
    assert H.lib().heddle_linear(C.byref(d), None, 0, None) == H.HEDDLE_E_DEVICE
