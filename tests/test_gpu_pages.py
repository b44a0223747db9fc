"""GPU: page tables and slot maps where their inputs are at the edge of what the entry
points take, against the oracle (whole numbers, equal)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2609_14717_amd as co  # noqa: E402
from oracle import serve8  # noqa: E402
from test_gpu_serve8 import Pool, dims, ints, np_, space, zero  # noqa: E402


def map_slots(start, pos0, table, rows, num_pages):
    """row_pos, row_dst (one entry more than the rows) and the status of one call."""
    d, status = dims(len(pos0), np.shape(table)[1], num_pages), zero()
    pos, dst = torch.full((2, rows + 1), 77, dtype=torch.int32, device="cuda")
    co.carryover_slot_map(d, rows, ints(start), ints(pos0), ints(table), pos, dst, status)
    assert int(pos[rows]) == int(dst[rows]) == 77
    return np_(pos)[:rows], np_(dst)[:rows], int(status)


# sequences on both sides of what fits in LDS; the start that falls at any place of a group
# of four rows, of a workgroup's threads, and the last one
FALLS = [(S, at) for S in (2, 37, 4096, 4097, 9000)
         for at in sorted({1, 2, 3, 6, 255, 256, 257, 4095, S}) if at <= S]


@pytest.mark.parametrize("S,at", FALLS)
@pytest.mark.parametrize("by", [1, 40])
def test_starts_that_decrease_give_no_row_a_slot(S, at, by):
    lengths = np.random.RandomState(S).randint(0, 4, S)
    lengths[at - 1] = 3
    start = np.concatenate([[0], np.cumsum(lengths)])
    table = np.arange(S * 4).reshape(S, 4)
    pos0 = np.arange(S) % 5
    rows = int(start[-1])
    want = serve8.slot_map(rows, start, pos0, table, 4, S * 4)
    got = map_slots(start, pos0, table, rows, S * 4)
    assert got[2] == want[2] == 0
    np.testing.assert_array_equal(got[1], want[1])
    start[at:] -= lengths[at - 1] + by                       # the sequence's end, before its start
    start += max(0, -int(start.min()))
    got = map_slots(start, pos0, table, rows, S * 4)
    want = serve8.slot_map(rows, start, pos0, table, 4, S * 4)
    assert got[2] == want[2] == co.CO_ERR_LENGTH
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def test_starts_that_decrease_more_than_once():
    start = list(range(0, 6000)) + [5, 900, 7] + list(range(9000, 12000))
    S = len(start) - 1
    pos, dst, st = map_slots(start, [0] * S, np.zeros((S, 600), int), 9000, 1)
    assert st == co.CO_ERR_LENGTH
    assert np.all(pos == 0) and np.all(dst == serve8.SKIP)


def test_as_many_rows_as_an_int_counts():
    """The row count's last workgroup lies past 2^31 rows; all but a few rows are padding."""
    rows = 2 ** 31 - 1
    d, status = dims(2, 2, 4), zero()
    pos, dst = (torch.full((rows + 1,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    start = [rows - 30, rows - 25, rows - 1]
    co.carryover_slot_map(d, rows, ints(start), ints([3, 0]), ints([[3, 1], [0, 2]]), pos, dst, status)
    wp, wd, st = serve8.slot_map(40, [10, 15, 39], [3, 0], [[3, 1], [0, 2]], 2, 4)   # the last forty
    assert int(status) == st == 0
    np.testing.assert_array_equal(np_(pos[-41:-1]), wp)
    np.testing.assert_array_equal(np_(dst[-41:-1]), wd)
    assert int(pos[-1]) == int(dst[-1]) == 77
    for a in range(0, rows - 40, 1 << 28):
        part = slice(a, min(a + (1 << 28), rows - 40))
        assert int(pos[part].count_nonzero()) == 0
        assert int((dst[part] != serve8.SKIP).count_nonzero()) == 0


# free slots of a server: runs of sequences without rows, in front, between and behind, where
# a thread's four rows begin on either side of the run
@pytest.mark.parametrize("idle", [1, 2, 3, 5, 8, 100, 2000, 4060, 6000])
@pytest.mark.parametrize("rows_of", [1, 2, 3, 4, 5])
def test_rows_on_both_sides_of_idle_sequences(idle, rows_of):
    r = np.random.RandomState(idle * 8 + rows_of)
    some = lambda: [rows_of] * 7  # noqa: E731
    lengths = [0] * 3 + some() + [0] * idle + some() + [0, 0] + some() + [0] * (idle // 3)
    S = len(lengths)
    start, pos0 = np.concatenate([[0], np.cumsum(lengths)]) + 1, r.randint(0, 60, S)
    table = r.permutation(S * 5).reshape(S, 5)
    rows = int(start[-1]) + 6
    want = serve8.slot_map(rows, start, pos0, table, 5, S * 5)
    got = map_slots(start, pos0, table, rows, S * 5)
    assert got[2] == want[2] == 0
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


@pytest.mark.parametrize("idle", [4000, 1 << 20])
def test_idle_sequences_are_not_walked(idle):
    """A walk of one sequence after the other is a chain of that many reads: 0.1 s for a
    million, 0.2 ms for 4000; the search takes a few microseconds, of which ten times as
    many are allowed."""
    start = ints(np.concatenate([[0, 3, 3 + 3], np.full(idle, 6), [9, 12]]))
    S = len(start) - 1
    d, status = dims(S, 1, 1), zero()
    pos, dst = torch.full((2, 12), 77, dtype=torch.int32, device="cuda")
    table, pos0 = torch.zeros((S, 1), dtype=torch.int32, device="cuda"), torch.zeros_like(start)
    times = []
    for _ in range(20):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        co.carryover_slot_map(d, 12, start, pos0, table, pos, dst, status)
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    assert np_(pos).tolist() == [0, 1, 2] * 4 and int(status) == 0
    assert min(times) < 100, times


# ------------------------------------------------------------- the page pool

# in one launch and in two
SIZES = pytest.mark.parametrize("max_pages", [8, 11000], ids=["one launch", "two"])


@SIZES
@pytest.mark.parametrize("want", [[0] * 6, [0, 30, 0, 5, 50, 0]])
def test_holdings_that_the_pool_cannot_have_change_nothing(want, max_pages):
    """More free and released pages than the pool has: before, the call took the holdings
    away and left a free count that every later call refuses."""
    p = Pool(6, max_pages, 20, 1)
    p.assign([20, 30, 40, 0, 50, 60])
    p.t["free_count"].fill_(20)                    # every page, and the held ones again
    before = {k: v.clone() for k, v in p.t.items()}
    p.status.zero_()
    co.carryover_assign_pages(p.d, ints(want), 0, p.t, p.status, p.ws)
    assert int(p.status) == co.CO_ERR_POOL
    assert all(torch.equal(p.t[k], before[k]) for k in before)
    p.t["free_count"].fill_(len(p.free))           # the count that it has: the pool serves on
    p.assign(want)
    p.assign([20, 30, 40, 0, 50, 60])


def test_free_and_released_pages_past_32_bits():
    S, P = 1024, 2 ** 21 - 1
    d, status = dims(S, P, 2 ** 27 - 1), zero()
    pool = dict(page_table=torch.full((S, P), 5, dtype=torch.int32, device="cuda"), held=ints([P] * S),
                free_pages=torch.full((2 ** 27 - 1,), 6, dtype=torch.int32, device="cuda"),
                free_count=ints([2 ** 27 - 1]))
    co.carryover_assign_pages(d, ints([0] * S), 0, pool, status, space(d, co.CO_WS_ASSIGN_PAGES))
    assert int(status) == co.CO_ERR_POOL
    assert int(pool["free_count"]) == 2 ** 27 - 1 and int(pool["held"].min()) == P
    assert int(pool["page_table"].min()) == 5 and int(pool["free_pages"].min()) == 6


@SIZES
@pytest.mark.parametrize("bad", [-1, 60, 2 ** 31 - 1, -2 ** 31])
def test_ids_of_no_page_are_reported_where_they_move(bad, max_pages):
    """In an entry that a sequence gives back (to another one, and to the free list), and
    in one that the free list gives."""
    full, some = [100, 90, 0, 60, 0, 0], [10, 90, 33, 60, 0, 70]
    for seq, place, then in ((0, 6, some), (0, 6, [0] * 6), (3, 1, [100, 90, 0, 0, 0, 0])):
        p = Pool(6, max_pages, 60, 1)
        p.assign(full)
        assert int(p.status) == 0
        p.table[seq][place] = bad
        p.t["page_table"].copy_(ints(p.table))
        p.assign(then)                                     # compares table, list and status
        assert int(p.status) == co.CO_ERR_PAGE_RANGE
        p.assign(full)                                     # and back again, exactly
        assert int(p.status) == co.CO_ERR_PAGE_RANGE and int(p.table[seq][place]) == bad
        p.assign([100, 90, 0, 60, 0, 0])                   # nothing moves: nothing to report
        assert int(p.status) == 0
    p = Pool(6, max_pages, 60, 1)
    p.free[-3] = bad
    p.t["free_pages"].copy_(ints(p.free))
    p.assign([1, 1, 0, 0, 0, 0])
    assert int(p.status) == 0
    p.assign([1, 1, 1, 0, 0, 0])
    assert int(p.status) == co.CO_ERR_PAGE_RANGE
