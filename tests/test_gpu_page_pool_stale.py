"""Compaction of a table with entries that the counts do not know: flagged and cleared wherever the page lies, so that no entry
names a page that the call has filled with another sequence's."""
import pytest

from tests.test_gpu_page_pool import Pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("locked", [False, True])
@pytest.mark.parametrize("stale", [1, 2, 3, 6, 11])
def test_entries_of_free_pages_are_flagged_and_cleared(stale, locked):
    p = Pair(4, 4, 12)
    p.reserve([(0, 0, 200), (1, 0, 130), (2, 0, 100)])               # pages 0 .. 3, 4 .. 6, 7 and 8
    p.fork([0], [3], [60])                                            # page 0 twice
    p.release([0, 1], [0, 128])                                       # free: 1, 2, 3, 6 and 9 .. 11; live: 0, 4, 5, 7, 8
    p.check()
    p.gpu.page_table[1, 3] = -2 - stale if locked else stale
    moves, live = p.ora.compact()
    p.gpu.compact([])
    assert live == 5 and [b for _, b in moves] == [1, 2, 3]
    assert p.gpu.status() == p.B.DEV_BAD_REFS and int(p.gpu.page_table[1, 3]) == -1
    p.check(moves, 6)
    p.gpu.dev_status.zero_()
    p.compact()                                                       # nothing moves, nothing is flagged any more
    assert p.gpu.status() == 0
