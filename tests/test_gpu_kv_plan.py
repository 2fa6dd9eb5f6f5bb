"""dgq_kv_plan where its inputs name pages that no cache has."""
import pytest

from dgq_testlib import gpu
from test_gpu_kv_cache import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("far", ["first", "wrapped", "largest", "negative"])
def test_pages_without_slots(page, far):
    """Page 2^32 / page + 3 times the page's size is the slot of page 3 in 32 bits."""
    _, b = gpu()
    last = (2 ** 31 - 1) // page  # the last page whose slots 31 bits hold
    p = {"first": last + 1, "wrapped": 2 ** 32 // page + 3, "largest": 2 ** 31 - 1, "negative": -2}[far]
    # the first request has begun page p and goes on to page 5, the second takes p and 6 from the free ones
    table = dev([[p, -1], [-1, -1]])
    start, lens, slots, used = b.kv_plan(dev([page - 1, 0]), dev([2, page + 1]), dev([5, p, 6]), table, page, page + 4)
    assert b.device_status() == 1
    assert table.tolist() == [[p, 5], [p, 6]] and start.tolist() == [0, 2, page + 3] and used.item() == 3
    assert slots.tolist() == [-1, 5 * page] + [-1] * page + [6 * page, -1]
    # the last page that has slots is a page like others
    _, _, slots, _ = b.kv_plan(dev([0]), dev([2]), dev([last]), dev([[-1]]), page, 2)
    assert b.device_status() == 0 and slots.tolist() == [last * page, last * page + 1]
