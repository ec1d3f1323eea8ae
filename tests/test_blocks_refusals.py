"""What the feed-forward block's entry points turn down on the host (no call reaches a kernel)."""
import os

import pytest

from paper_2011_13824_amd import lirpa

P, Q, R = 0x10000, 0x20000, 0x30000  # stand for device pointers: only their alignment is looked at


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lirpa.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return lirpa.load()


@pytest.mark.parametrize("sum_at,lds", [(P, 9), (P, 12), (Q, 8), (Q, 10)])
def test_norm_sum_in_place_with_another_row_distance(L, sum_at, lds):
    """x has rows of 8, res of 9: a sum in either's buffer with other rows would be written over
    rows that are still to be read."""
    assert L.lirpa_norm_forward(lirpa.F32, 4, 8, P, 8, Q, 9, R, 1e-5, sum_at, lds, None, 0, None,
                                None, None) == lirpa.LIRPA_EINVAL
    assert "sum is the buffer of" in lirpa.lirpa_last_error()


@pytest.mark.parametrize("dh,lddh", [(P, 9), (P, 12), (Q, 8), (Q, 10)])
def test_norm_gradient_in_place_with_another_row_distance(L, dh, lddh):
    assert L.lirpa_norm_backward(lirpa.F32, 4, 8, P, 8, Q, 9, R, 8, R, R, dh, lddh, None, None, 0,
                                 None) == lirpa.LIRPA_EINVAL
    assert "dh is the buffer of" in lirpa.lirpa_last_error()
