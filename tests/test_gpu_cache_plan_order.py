"""Which requests the plan of the 4-bit cache serves where a row of the table is full and the pool is short at once: a full row asks for nothing, a need that the pool
cannot fill counts for the requests behind it."""
import numpy as np
import pytest

from test_gpu_cache_plan import Served

pytestmark = pytest.mark.gpu


def served(held, new, free, page, max_pages):
    """The rule as a sentence about each request: (full, the pages it takes)."""
    need = [-(-(h + n) // page) - -(-h // page) if n >= 0 else 0 for h, n in zip(held, new)]
    row = [n < 0 or -(-(h + n) // page) <= max_pages for h, n in zip(held, new)]
    full, taken = [], []
    for i in range(len(held)):
        ok = row[i] and (need[i] == 0 or sum(w for w, r in zip(need[:i + 1], row) if r) <= free)
        taken.append(need[i] if ok else 0)
        if not ok:
            full.append(i)
    return full, taken


def test_a_full_row_asks_for_nothing(dsn):
    s = Served(dsn, 4, 96, 16, 12, 4)
    assert s.step([64, 16, 16, 0]) == ([], [])                     # 4 + 1 + 1 pages of 12: 6 left
    assert s.step([96, 48, 48, 0]) == ([0], [])                    # the first would need 6 more and has no room in its row: 3 + 3 for the others
    assert s.held == [64, 64, 64, 0] and s.free == 0


def test_a_need_that_the_pool_cannot_fill_counts(dsn):
    s = Served(dsn, 5, 96, 16, 12, 5)
    assert s.step([80, 16, 16, 0, 0]) == ([], [])                  # 5 + 1 + 1: 5 left
    assert s.step([16, 64, 32, 16, 0]) == ([0, 2, 3], [])          # row full; 4 of 5; 2 more than is left; 1 behind a need that counts
    assert s.held == [80, 80, 16, 0, 0] and s.free == 1
    assert s.step([16, 16, 0, 16, 1]) == ([0, 1, 4], [])           # two full rows in front of the one that gets the last page
    assert s.held == [80, 80, 16, 16, 0] and s.free == 0


@pytest.mark.parametrize("B,R,page,n_pages,max_pages", [(7, 12, 16, 8, 2), (40, 7, 16, 25, 1), (33, 200, 16, 150, 9), (700, 90, 16, 1900, 5), (1500, 4, 16, 900, 1),
                                                       (2100, 70, 32, 3000, 3)])
def test_full_rows_and_a_short_pool_together(dsn, B, R, page, n_pages, max_pages):
    g = np.random.default_rng(B)
    s = Served(dsn, B, R, page, n_pages, max_pages)
    rows = pools = 0
    for _ in range(10):
        new = g.integers(0, R + 1, size=B)
        new[g.random(B) < 0.2] = -1
        want, taken = served(s.held, new.tolist(), s.free, page, max_pages)
        held, free = list(s.held), s.free
        full, bad = s.step(new.tolist())                           # against the plan made request by request
        assert not bad and full == want
        assert s.free == free - sum(taken) + sum(-(-h // page) for h, n in zip(held, new) if n < 0)
        over = {i for i in full if -(-(held[i] + new[i]) // page) > max_pages}
        rows += len(over)
        pools += len(set(full) - over)
    assert rows and pools                                           # both reasons came up
