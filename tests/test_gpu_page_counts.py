"""Page updates whose reference counts are not what the tables list: counts that are too low are reported and taken for the number
of listings, so that no page is handed out that a table lists; counts that are too high hold their page."""
import numpy as np
import pytest

from paper_2609_34977_gb300 import _native as N
from tests.test_gpu_pages import _check_update, _pool_of, _ref_of, _run_update, _table, _update, pytestmark  # noqa: F401


def _low(ref, table, lens, parent, grow, page, g=1, d=64, pool=None):
    """An update with counts that are too low: as with the right ones, and reported."""
    table = np.asarray(table, np.int32)
    pool = _pool_of(2, len(ref), page, g, d) if pool is None else pool
    before = pool.clone()
    right = np.maximum(ref, _ref_of(table, lens, page, len(ref)))
    assert (right != np.asarray(ref)).any()
    w_ref, w_table, w_len, moved, short = _update(right, table, lens, parent, grow, page)
    assert not short
    r, t, ln, status = _run_update(pool, ref, table, lens, parent, grow, g, d)
    assert status == N.SPD_EINVAL
    np.testing.assert_array_equal(t, w_table)
    np.testing.assert_array_equal(np.maximum(r, 0), w_ref)  # (0 or less: free)
    np.testing.assert_array_equal(ln, w_len)
    for a, b, rows in moved:
        before[:, b, :rows] = before[:, a, :rows]
    assert (pool == before).all()


TABLE = [[0, 1, -1, -1], [2, -1, -1, -1], [3, 1, -1, -1]]
LENS = [20, 16, 22]


@pytest.mark.parametrize("parent,grow", [
    ([0, 1, 2], [1, 1, 20]),        # every sequence goes on once: no count changes
    ([0, 0, 1, 2, 2], [1, 3, 1, 1, 0]),
    ([1, 1], [1, 1]),               # two end
    ([-1, 2], [40, 1]),
    ([-1], [16]),                   # all end
    ([0, 1, 2], [0, 0, 0]),         # nobody needs a page
])
@pytest.mark.parametrize("ref", [[0] * 16, [1, 1, 1, 1] + [0] * 12, [1, 2, 0, 1] + [0] * 12, [-5, 0, 1, 1] + [0] * 12])
def test_counts_that_are_too_low(ref, parent, grow):
    _low(ref, TABLE, LENS, parent, grow, 16)


def test_a_page_that_a_table_lists_twice():
    _low([1] + [0] * 8, [[0, 0, -1]], [30], [0, 0], [1, 5], 16)


@pytest.mark.parametrize("pages", [700, 15000])  # with the counters in shared memory, and in the workspace
@pytest.mark.parametrize("seed", range(3))
def test_many_low_counts(pages, seed):
    page, r = 16, np.random.default_rng(seed)
    lens = [int(x) for x in r.integers(1, 100, 60)]
    table, n = _table(r, lens, page, extra=pages - sum(-(-x // page) for x in lens), width=9)
    assert n == pages
    table[5, :3] = table[4, :3]  # (sequences share pages)
    table[6] = table[7]
    lens[6] = lens[7]
    lens[4] = lens[5] = max(48, lens[4], lens[5])
    ref = np.maximum(0, _ref_of(np.where(table < pages, table, 0), lens, page, pages) - (r.random(pages) < 0.3))
    table = np.where(table < pages, table, 0)
    parent = [int(x) for x in r.integers(0, 60, 100)]
    _low(ref.astype(np.int32), table, lens, parent, [int(x) for x in r.integers(0, 20, 100)], page)


def test_counts_that_are_too_high_hold_their_page():
    page = 16
    table = np.asarray(TABLE, np.int32)
    _check_update(_pool_of(2, 16, page, 1, 64), [3, 4, 2, 2] + [0] * 11 + [1], table, LENS, [0, 0, 1, 2], [1, 20, 3, 1], 1, 64, page)
    _check_update(_pool_of(2, 16, page, 1, 64), [3, 4, 2, 2] + [0] * 11 + [1], table, LENS, [-1], [20], 1, 64, page)
