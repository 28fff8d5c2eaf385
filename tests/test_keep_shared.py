"""Keeping drafted tokens in rows that share pages, the oracle on the CPU: a row never comes to end inside a page that another row has
as well, since its next tokens would be written there."""
import numpy as np

from oracle import drafts, kv_pages


def shared(extra=0):
    """Row 0 has 96 tokens, its last 46 drafted; row 1 is forked from it behind them, so that all three pages are shared."""
    c = kv_pages.Cache(np.full((3, 2, 6), -1), [0, 0, 0], np.zeros(40, int), (np.arange(40 * 32).reshape(40, 32, 1).copy(),))
    c.extend([0], [96 + extra])
    c.fork([0], [1])
    return c


def test_rows_do_not_end_inside_a_page_of_another():
    for path in ([0], [0, 1], [], list(range(45))):  # nothing moves: places 0, 1, ..
        c = shared()
        before = c.table.copy(), c.refs.copy()
        drafts.keep(c, [0], [0, 46], path + [-1] * (46 - len(path)), [len(path)])
        assert c.lens.tolist() == [96, 96, 0] and np.array_equal(c.table, before[0]) and np.array_equal(c.refs, before[1])


def test_rows_may_end_where_a_shared_page_does():
    c = shared()
    drafts.keep(c, [0], [0, 46], list(range(14)) + [-1] * 32, [14])
    assert c.lens.tolist() == [64, 96, 0] and c.table[0, :, 2].tolist() == [-1, -1]
    assert c.refs[c.table[1, :, 2]].tolist() == [1, 1] and c.refs[c.table[1, :, 1]].tolist() == [2, 2]
    c = shared()
    drafts.keep(c, [0], [0, 46], list(range(46)), [46])  # (all of them: the row ends where it did)
    assert c.lens[0] == 96
    c = shared(extra=4)  # a part page at the end, which the fork has a copy of
    drafts.keep(c, [0], [0, 4], [0, 1, -1, -1], [2])
    assert c.lens.tolist() == [98, 100, 0]
    # the other row gone, the page is the row's own
    c = shared()
    c.free([1])
    drafts.keep(c, [0], [0, 46], [0] + [-1] * 45, [1])
    assert c.lens[0] == 51


def test_what_a_row_grows_by_leaves_its_fork_as_it_is():
    for path in ([0], [], list(range(14)), [0, 1, 40]):
        c = shared()
        mine = c.pools[0].copy()
        drafts.keep(c, [0], [0, 46], path + [-1] * (46 - len(path)), [len(path)])
        start = int(c.lens[0])
        c.extend([0], [start + 20])
        for p in range(start, start + 20):  # what an append does
            for h in range(2):
                c.pools[0][c.table[0, h, p // 32], p % 32] = -7
        for p in range(96):
            for h in range(2):
                at = c.table[1, h, p // 32]
                assert c.pools[0][at, p % 32] == mine[at, p % 32]
