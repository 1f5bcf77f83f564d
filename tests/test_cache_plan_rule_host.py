"""The oracle's plan of the 4-bit cache against the rule of service said of each request by itself, with full rows of the table and a short pool.  No GPU."""
import numpy as np
import pytest

from oracle import dsn_oracle as O
from test_gpu_cache_plan_order import served


@pytest.mark.parametrize("B,R,page,N,max_pages", [(7, 12, 16, 8, 2), (40, 7, 16, 25, 1), (33, 200, 16, 150, 9), (700, 90, 16, 1900, 5)])
def test_who_is_served(B, R, page, N, max_pages):
    g = np.random.default_rng(B)
    held, table, ring, first, free = [0] * B, [[] for _ in range(B)], list(range(N)), 0, N
    rows = pools = 0
    for _ in range(12):
        new = g.integers(0, R + 1, size=B)
        new[g.random(B) < 0.2] = -1
        want, taken = served(held, new.tolist(), free, page, max_pages)
        over = {i for i in range(B) if -(-(held[i] + new[i]) // page) > max_pages}
        _, held, table, _, ring, first, after, full, bad = O.cache_plan(held, new.tolist(), table, ring, first, free, page, max_pages, R)
        assert full == want and not bad
        free, table = after, [t[:-(-h // page)] for t, h in zip(table, held)]
        owned = [p for t in table for p in t]
        assert sorted(owned + [ring[(first + j) % N] for j in range(free)]) == list(range(N))     # every page once
        rows += len(over)
        pools += len(set(full) - over)
    assert rows and pools
