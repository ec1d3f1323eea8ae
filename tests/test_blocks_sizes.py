"""Sizes that the feed-forward block's entry points report, over many sizes (no GPU)."""
import ctypes
import os

import pytest

from paper_2011_13824_amd import lirpa

P = 0x10000  # stands for a device pointer: only its alignment is looked at


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lirpa.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return lirpa.load()


@pytest.mark.parametrize("dtype", [lirpa.F32, lirpa.BF16, lirpa.F16])
@pytest.mark.parametrize("D,F", [(64, 96), (1, 1), (256, 4288), (1001, 2731), (1024, 2752),
                                 (2048, 5504), (4096, 10944), (192, 42688), (5504, 2048)])
@pytest.mark.parametrize("backward", [0, 1])
def test_a_workspace_for_many_rows_holds_fewer(L, dtype, D, F, backward):
    block = ctypes.byref(lirpa.lirpa_ffn(dtype, 1, D, F, P, P, P, D, D, F))
    rows = [*range(2600), *range(2600, 20000, 37), *range(20000, 1 << 17, 997), 1 << 20, 1 << 30]
    last = 0
    for r in rows:
        need = L.lirpa_ffn_workspace_bytes(block, r, backward)
        assert need >= last, (r, need, last)
        last = need
