"""Pages and slots of the 4-bit cache planned on the GPU, against the same plan made request by request."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from cache_util import up
from gpu_util import DEV

pytestmark = pytest.mark.gpu


class Served:
    """A cache's bookkeeping on the device and the oracle's beside it."""

    def __init__(self, dsn, B, R, page, n_pages, max_pages):
        self.dsn, self.ctx, self.B, self.R, self.page, self.max_pages = dsn, dsn.Context(0), B, R, page, max_pages
        self.d = dsn.make_cache_desc(R, 2, 64, [2], page=page, n_pages=n_pages, max_pages=max_pages)
        i32 = lambda *shape: torch.full(shape, -7, dtype=torch.int32, device=DEV)
        self.t = dict(table=i32(B, max_pages), lengths=i32(B), placed=i32(B), slots=i32(B, R), pool=i32(n_pages), pool_state=i32(2))
        self.c = dsn.make_cache(**self.t)
        dsn.dsn_cache_reset(self.ctx, self.d, self.c, B)
        self.held, self.table, self.ring, self.first, self.free = [0] * B, [[] for _ in range(B)], list(range(n_pages)), 0, n_pages

    def step(self, new, status=True, **kw):
        before = self.t["table"].cpu().numpy().copy()
        self.dsn.dsn_cache_plan(self.ctx, self.d, self.c, self.B, up(new), **kw)
        code, detail = self.ctx.get_status()
        placed, lengths, table, slots, ring, first, free, full, bad = O.cache_plan(self.held, new, self.table, self.ring, self.first, self.free,
                                                                                  self.page, self.max_pages, self.R)
        got = {k: v.cpu().numpy() for k, v in self.t.items()}
        lengths_got = kw["lengths_out"].cpu().numpy() if "lengths_out" in kw else got["lengths"]
        state_got = kw["pool_state_out"].cpu().numpy() if "pool_state_out" in kw else got["pool_state"]
        assert np.array_equal(got["placed"], placed)
        assert np.array_equal(lengths_got, lengths)
        assert np.array_equal(got["slots"], np.array(slots).reshape(self.B, self.R))
        assert list(state_got) == [first, free]
        for j in range(free):
            e = (first + j) % len(ring)
            assert got["pool"][e] == ring[e]
        for i in range(self.B):
            n = -(-lengths[i] // self.page) if i not in bad else 0
            assert list(got["table"][i, :n]) == table[i][:n]
            assert np.array_equal(got["table"][i, n:], before[i, n:])              # entries behind stay as they were
        # a page is in the ring or with one request
        owned = [p for i in range(self.B) if i not in bad for p in table[i][:-(-lengths[i] // self.page)]]
        if not bad:
            assert sorted(owned + [ring[(first + j) % len(ring)] for j in range(free)]) == list(range(len(ring)))
        if full or bad:
            assert code in ([self.dsn.ERR_CACHE_FULL] if full else []) + ([self.dsn.ERR_BAD_INDEX] if bad else []) and detail in full + bad
        else:
            assert code == 0
        if "lengths_out" not in kw:
            self.held, self.table, self.ring, self.first, self.free = lengths, table, ring, first, free
        return full, bad


@pytest.mark.parametrize("B,R,page,n_pages,max_pages", [(1, 1, 16, 3, 3), (5, 7, 16, 40, 9), (64, 1, 16, 500, 20), (33, 300, 48, 400, 30),
                                                       (40, 700, 16, 3000, 200), (1500, 3, 32, 2000, 4), (2049, 130, 128, 9000, 7)])
def test_serving_a_while(dsn, B, R, page, n_pages, max_pages):
    g = np.random.default_rng(B + R)
    s = Served(dsn, B, R, page, n_pages, max_pages)
    seen_full = False
    for _ in range(14):
        new = g.integers(0, R + 1, size=B)
        new[g.random(B) < 0.15] = -1
        new[g.random(B) < 0.1] = 0
        new = np.array([n if n < 0 or s.held[i] + n <= max_pages * page else -1 for i, n in enumerate(new)])
        full, _ = s.step(new.tolist())
        seen_full |= bool(full)
    if n_pages < B:
        assert seen_full


def test_pool_runs_dry_and_fills_again(dsn):
    s = Served(dsn, 6, 64, 16, 10, 8)
    assert s.step([64, 64, 32, 0, 0, 0]) == ([], [])           # 4 + 4 + 2 pages
    assert s.step([0, 0, 1, 16, 0, 0]) == ([2, 3], [])         # both need a page
    assert s.step([-1, 0, 16, 0, 0, 0]) == ([2], [])           # pages given back now come with the next call
    assert s.step([0, 0, 16, 48, 1, 0]) == ([4], [])
    assert s.step([0, 64, 0, 0, 0, 0]) == ([1], [])
    assert s.step([-1] * 6) == ([], [])
    assert s.free == 10 and s.held == [0] * 6


def test_row_of_the_table_is_full(dsn):
    s = Served(dsn, 3, 40, 16, 20, 4)
    assert s.step([40, 24, 40]) == ([], [])
    assert s.step([24, 40, 25]) == ([2], [])                   # 64 tokens fit, 65 do not
    assert s.step([1, 0, 24]) == ([0], [])


def test_numbers_out_of_range_change_nothing(dsn):
    s = Served(dsn, 5, 8, 16, 20, 4)
    s.step([8, 3, 8, 8, 8])
    assert s.step([9, -2, 5, 2 ** 31 - 1, -2 ** 31]) == ([], [0, 1, 3, 4])
    s.t["lengths"][1] = -1
    s.t["lengths"][2] = 65
    s.held[1], s.held[2] = -1, 65
    assert s.step([2, 2, 2, -1, 2])[1] == [1, 2]


def test_results_beside_the_cache_and_replay(dsn):
    s = Served(dsn, 70, 90, 32, 600, 12)
    g = np.random.default_rng(0)
    for _ in range(3):
        s.step(g.integers(0, 91, size=70).tolist())
    new = g.integers(-1, 91, size=70)
    out = dict(lengths_out=torch.zeros(70, dtype=torch.int32, device=DEV), pool_state_out=torch.zeros(2, dtype=torch.int32, device=DEV))
    s.step(new.tolist(), **out)
    first = {k: v.clone() for k, v in {**s.t, **out}.items()}
    s.step(new.tolist(), **out)                                # nothing that is read was changed: the same again
    assert all(torch.equal(v, first[k]) for k, v in {**s.t, **out}.items())
    # in place, captured: every replay is the next step
    one = up([1] * 70)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        dsn.dsn_cache_plan(s.ctx, s.d, s.c, 70, one)
    before = s.t["lengths"].clone()
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert s.ctx.get_status()[0] == 0
    assert torch.equal(s.t["lengths"], before + 5)


def test_no_requests(dsn):
    s = Served(dsn, 1, 1, 16, 3, 3)
    dsn.dsn_cache_plan(s.ctx, s.d, s.c, 0, None)
    assert s.t["pool_state"].tolist() == [0, 3] and s.ctx.get_status()[0] == 0
