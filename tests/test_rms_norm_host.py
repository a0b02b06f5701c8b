"""Sizes at the border of what one launch covers: refused as shapes, not by a launch that fails.  No GPU needed (as in
tests/test_e4m3_host.py, every call is refused before its pointers are looked at)."""
import pytest

from tests.test_e4m3_host import ALIGN, P, SHAPE, norm, t8

LANES = (1 << 32) - 1                                  # of a launch


@pytest.mark.parametrize("C", [8208, 9216, 9232, 16384])
def test_rms_norm_rows_of_one_launch(C):
    """A row takes a workgroup of 64 lanes for 1024 elements."""
    most = LANES // (64 * -(-C // 1024))
    assert most < LANES // 512
    for T, status in ((most + 1, SHAPE), (LANES // 512, SHAPE), (most, ALIGN)):        # (ALIGN: what is refused next, the weight's address)
        assert norm(T=T, C=C, ld=C, w=P + 2, out=t8(T, C)) == status, T


@pytest.mark.parametrize("C", [16, 1024, 1040, 8192])
def test_rms_norm_rows_of_one_launch_up_to_512_lanes(C):
    for T, status in ((LANES // 512 + 1, SHAPE), (LANES // 512, ALIGN)):
        assert norm(T=T, C=C, ld=C, w=P + 2, out=t8(T, C)) == status, T
