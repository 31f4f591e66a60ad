"""A product whose depth is split over workgroups (no kernel is launched): every part has some of the depth.  One without would read its
scales from an address that is no whole word, write zeros and have them read back."""
import pytest

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
