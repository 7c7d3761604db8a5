"""Host checks of a step's slot map and of attention's scale on the CPU (fake addresses: refused
before any device work)."""
import pytest

from paper_2410_18701_amd import baton as B
from tests.test_paged_abi import M, attn, desc, status


@pytest.mark.parametrize("map_ld", [0, 4, -1, -(1 << 62), (1 << 40) + 1, (1 << 62), (1 << 63) - 1])
def test_row_distances_refused(map_ld):
    assert status(B.baton_paged_step, desc(), 0, M, M, 5, map_ld) == B.BATON_EINVAL


@pytest.mark.parametrize("scale", [2.0 ** 127 * 1.5, -3.4e38, float("-inf")])
def test_scales_refused(scale):
    """Times log2 e they are infinite in fp32."""
    assert attn(scale=scale) == B.BATON_EINVAL
