"""Rings of free pages that are none, and pages that the pool has not: what `cache_reserve` then says and leaves."""
import pytest

from test_gpu_refused import bounds_reported, reserve, select  # noqa: F401 (a fixture)
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state", [[5, 1], [-1, 1], [0, 4], [0, -2]])
def test_a_ring_that_is_none_takes_nothing_back(select, state):  # noqa: F811
    """A request that would give pages back still holds them, and its length says so."""
    s = select.Selector(3, 8, 8, 4, 4, 64, "bf16")
    table, free = i32([[0, -1], [1, 0], [2, -1]]), i32([2, -1, -1])
    g, st, sl = reserve(s, table, [16, 32, 10], [17, 0, 12], free, state, [1, 0, 2])
    assert bounds_reported(select, s)
    assert g == [16, 32, 12] and st == state and sl == [-1, 42, 43]  # the third needs no other page
    assert table.tolist() == [[0, -1], [1, 0], [2, -1]] and free.tolist() == [2, -1, -1]
    # the pages go back by the next call, with a ring that is one
    g, st, _ = reserve(s, table, g, [16, 0, 12], free, [0, 1], [0, 0, 0])
    assert g == [16, 0, 12] and st == [0, 3] and free.tolist() == [2, 1, 0]
    s.check_device()
    s.close()


def test_an_entry_that_is_no_page_goes_round_the_ring(select):  # noqa: F811
    """It is counted and handed on like a page, reported each time, and its tokens have no slot."""
    s = select.Selector(2, 8, 8, 4, 4, 64, "bf16")
    table, free = i32([[0, -1, 9], [-1, -1, -1]]), i32([2, -1, -1, -1])
    g, st, _ = reserve(s, table, [48, 0], [16, 0], free, [0, 1], [0, 0])
    assert bounds_reported(select, s)
    assert g == [16, 0] and st == [0, 3] and free.tolist() == [2, -1, 9, -1]
    g, st, sl = reserve(s, table, [16, 0], [16, 40], free, st, [0, 40])
    assert bounds_reported(select, s)
    assert g == [16, 40] and st == [3, 0] and table[1].tolist() == [2, -1, 9]
    assert sl == list(range(32, 48)) + [-1] * 24
    s.close()
