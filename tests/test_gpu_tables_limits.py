"""Counts of free pages that cannot be (needs an MI355X)."""

import pytest

from tests.test_gpu_tables import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("count", [7, 10 ** 6, 2 ** 31 - 1])
def test_more_free_pages_than_there_are(count, packed):
    """All of the list then, the entries behind the true count among them: whatever they hold."""
    print("[case] too many", count, packed, flush=True)
    table, free, true = make(3, 4, 8, [0, 0, 0], 6, seed=6)
    assert len(free) == true == 6
    check(table, [0, 0, 0], [20, 3, 30], free, count, 8, 40, 0, packed)
    table, free, true = make(3, 4, 8, [9, 9, 9], 6, seed=6)
    assert len(free) == 12 and true == 6
    check(table, [9, 9, 9], [3, 10, 2], free, max(count, 13), 8, 40, 0, packed)
    table, free, true = make(3, 4, 8, [9, 9, 9], 6, seed=6)
    check(table, [9, 9, 9], [3, -1, 2], free, max(count, 13), 8, 40, 0, packed)     # pages that come back find no room
