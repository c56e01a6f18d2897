"""Page calls at sizes that take other paths: pools beyond the last-level cache, whose pages move past it, and tables
so wide that one sum of what sequences lack could overflow."""
import pytest
import torch

import paper_2608_02391_amd as cp
from test_gpu_pages import Rig, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("order", ["hnd", "nhd", "apart"])
@pytest.mark.parametrize("pages", [4096, 4097, 4500])
def test_compaction_of_a_pool_beyond_the_caches(order, pages):
    """Pages of 64 KiB: 4,096 of them are 256 MiB, the rule's limit."""
    print(f"large compaction pages={pages} {order}", flush=True)
    r = Rig(40, 120, pages, 16, layers=2, heads=4, dim=128, order=order)
    lens = [1 + (731 * s) % (100 * 16) for s in range(40)]
    r.reserve(list(range(40)), lens)
    r.free(list(range(0, 40, 3)))
    empty = [s for s in range(40) if r.m.lengths[s] == 0]
    live = [s for s in range(40) if r.m.lengths[s] > 0]
    r.fork([live[5], live[7]], empty[:2])
    r.free([live[5], live[0]])
    r.compact()
    r.compact()                                       # nothing is left to move


@pytest.mark.parametrize("width", [(1 << 20) - 1, 1 << 20, (1 << 20) + 5])
def test_reservations_through_wide_tables(width):
    """Pages of one token, sequences that lack more than 65,536 of them; too few; growth from there."""
    print(f"wide table width={width}", flush=True)
    r = Rig(4, width, (1 << 21) + 77, 1, layers=1, heads=1, dim=8)
    r.reserve([2, 0, 1], [700001, 3, width])
    assert int(r.status) == cp.PAGES_OK
    r.reserve([3, 2], [width, 700002])                # what is left does not do
    assert int(r.status) == cp.PAGES_SHORT
    r.reserve([3], [width + 1])
    assert int(r.status) == cp.PAGES_BAD_SEQUENCE
    r.reserve([3, 0, 2], [65536, 65540, 700003])
    assert int(r.status) == cp.PAGES_OK
    r.free([1, 2])
    r.reserve([1], [131071])
    assert int(r.status) == cp.PAGES_OK
