"""A step's slot map in rows far apart."""
import pytest
import torch

from paper_2410_18701_amd import baton as B
from paper_2410_18701_amd.paged import PagedCache
from tests.test_gpu_paged import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("map_ld", [5, 7, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1])
def test_rows_apart(map_ld):
    """Distances past 31 and 32 bits: the rows lie there and nothing else is written."""
    c = PagedCache(1, 2, 2, 1, 64, 8, 4, page=32, width=5)
    c.begin(i32([30, 0]))
    places = torch.full((map_ld + 6,), -7, dtype=torch.int32, device="cuda")
    B.baton_paged_step(c.desc, i32([30, 0]), i32([3, 5]), places, 5, map_ld, None, torch.cuda.current_stream())
    assert places[:5].tolist() == [30, 31, 32, -1, -1]
    assert places[map_ld:map_ld + 5].tolist() == [64, 65, 66, 67, 68]
    places[:5], places[map_ld:map_ld + 5] = -7, -7
    assert int(torch.stack([(x != -7).any() for x in places.split(1 << 30)]).sum()) == 0
