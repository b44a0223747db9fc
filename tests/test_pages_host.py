"""Page tables and slot maps without a GPU: pins of the oracle's answers to inputs that the
entry points report."""
import numpy as np

from oracle import SKIP, serve8


def test_starts_that_decrease_give_no_row_a_slot():
    table = [[0, 1], [2, 3], [4, 5]]
    for start in ([0, 6, 2, 8], [3, 0, 4, 8], [0, 4, 8, 7]):
        pos, dst, st = serve8.slot_map(8, start, [0, 0, 0], table, 2, 6)
        assert st == serve8.ERR_LENGTH
        assert pos.tolist() == [0] * 8 and dst.tolist() == [SKIP] * 8
    assert serve8.slot_map(8, [0, 4, 4, 8], [0, 0, 0], table, 2, 6)[2] == serve8.OK


def test_holdings_that_the_pool_cannot_have_change_nothing():
    table = np.array([[0, 1], [2, 3]])
    t, held, free, st = serve8.assign_pages([0, 16], 0, table, [2, 2], [4, 5, 6], 2, 5)
    assert st == serve8.ERR_POOL and held == [2, 2] and free == [4, 5, 6]
    np.testing.assert_array_equal(t, table)
    t, held, free, st = serve8.assign_pages([0, 16], 0, table, [2, 2], [4, 5], 2, 5)
    assert st == serve8.OK and held == [0, 1] and free == [4, 5, 3, 1, 0]


def test_ids_of_no_page_are_reported_where_they_move():
    table = np.array([[0, -1], [2, 3]])
    t, held, free, st = serve8.assign_pages([1, 0], 0, table, [2, 2], [4, 9], 2, 6)
    assert st == serve8.ERR_PAGE_RANGE and held == [1, 0] and free == [4, 9, 3, 2, -1]
    t, held, free, st = serve8.assign_pages([17, 32], 0, t, held, free, 2, 6)
    assert st == serve8.ERR_PAGE_RANGE and held == [2, 2] and free == [4, 9]
    np.testing.assert_array_equal(t, table)
    t, held, free, st = serve8.assign_pages([1, 32], 0, [[0, 1], [2, 3]], [2, 2], [4, 9], 2, 6)
    assert st == serve8.OK                        # the free list's 9 stays where it is
