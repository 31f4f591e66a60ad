"""A product whose depth is split over workgroups (no kernel is launched): every part has some of the depth.  One without would read its
scales from an address that is no whole word, write zeros and have them read back."""
import ctypes as C

import pytest
import torch

from paper_2512_22804_amd import mx

STAGE = 256                             # of the depth: what a part is a whole number of


def parts(m, n, k):
    """Parts of the depth, 1: not split."""
    one = m * (-(-n // 4) * 4) * 4
    size = mx.mor_mx_product_workspace_bytes(m, n, k)
    assert size % one == 0
    return max(size // one, 1)


@pytest.mark.parametrize("m, n, k", [(100, 257, 8200), (128, 128, 9000), (70, 100, 4096), (300, 130, 6000), (128, 4096, 14336), (100, 33, 5000),
                                     (65, 65, 100000), (128, 512, 7777), (90, 200, 12345)])
def test_no_part_is_empty(m, n, k):
    stages = -(-k // STAGE)
    each = -(-stages // parts(m, n, k))
    assert (parts(m, n, k) - 1) * each < stages


def test_these_are_split():
    assert all(parts(*size) > 1 for size in ((100, 257, 8200), (128, 128, 9000), (128, 4096, 14336), (65, 65, 100000)))


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: nothing may be launched")
def test_no_depth_at_all():
    """A product over the experts' depth without a slot: nothing to split.  Without a GPU the launch fails; the plan before it must not divide
    by the number of stages."""
    order = mx.MorExpertOrder(0, 2, 3, 128, 0, 0, 1 << 40, None, None)
    op = mx.MorMxOperand(1 << 40, 16, 1 << 40, 4, 0, 0)
    status = mx.load().mor_mx_product_depth(8, 8, C.byref(op), C.byref(op), C.byref(order), 1 << 40, 8, 64, 0, None)
    assert status in (0, 6)
