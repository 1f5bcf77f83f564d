"""How exact attention over the 4-bit cache is: the bound of what each form rounds, the share of outputs that are not the formula's own rounding, the norm of the error."""
import numpy as np
import pytest

from cache_bounds import FEW_SHARE, MANY_SHARE, RELATIVE, few_rows, many_rows, relative, share_off
from cache_util import Pages
from oracle import dsn_oracle as O
from test_gpu_cache_attention import attend

pytestmark = pytest.mark.gpu
SENTINEL = 776.0


def check(pages, heads, group, idx, R, placed, x, got, scale=0.0, window=0, statistics=True):
    many = R * group > 32
    bound_of, sc = many_rows if many else few_rows, scale or pages.D ** -0.5
    outs, refs = [], []
    for i, L in enumerate(pages.lengths):
        n = R if placed is None else placed[i]
        assert np.all(got[i, n:] == SENTINEL) and np.all(got[i, :, heads[idx[i]]:] == SENTINEL)
        for h in range(heads[idx[i]]):
            k, v = pages.kv(i, h)
            for e in range(group):
                q = x[i, :n, h, e]
                ref, p = O.cache_attention(q, k, v, sc, L - n, window)
                err, bound = np.abs(got[i, :n, h, e] - ref), bound_of(pages, i, h, q, p, ref, sc)
                assert np.all(err <= bound), (i, h, e, float((err / bound).max()))
                outs.append(got[i, :n, h, e].ravel())
                refs.append(ref.ravel())
    out, ref = np.concatenate(outs), np.concatenate(refs)
    if statistics:
        assert out.size > 1000
        assert share_off(out, ref) <= (MANY_SHARE if many else FEW_SHARE)
        assert relative(out, ref) <= RELATIVE


CASES = [
    # D, H, group, page, heads, R, order, lengths, placed
    (64, 12, 1, 16, [12], 1, "input", [197, 64, 1], None),
    (64, 6, 1, 64, [3, 6], 1, "grouped", [30, 500, 64, 1999, 129, 16, 17], None),
    (128, 4, 4, 16, [4], 1, "input", [3000, 700, 65], None),
    (128, 2, 8, 256, [2], 1, "input", [9000, 300], None),
    (64, 4, 2, 32, [2, 4], 5, "grouped", [700, 64, 1200, 40], [5, 3, 5, 1]),
    (128, 2, 3, 48, [2], 4, "input", [900, 100], None),
    (64, 2, 17, 16, [2], 1, "input", [800, 90], None),
    (128, 2, 16, 16, [1, 2], 2, "grouped", [700, 64, 2000], None),
    (64, 2, 1, 16, [2], 32, "input", [600, 32], None),
    (64, 2, 11, 16, [2], 3, "input", [700, 130], None),
    (128, 2, 1, 64, [2], 33, "input", [2000, 400], [33, 20]),
    (64, 3, 4, 48, [2, 3], 64, "grouped", [64, 900, 300], None),
    (128, 2, 4, 16, [2], 130, "input", [130, 1700], None),
    (64, 1, 2, 16, [1], 300, "input", [300, 1200], [300, 257]),
]


@pytest.mark.parametrize("D,H,group,page,heads,R,order,lengths,placed", CASES)
@pytest.mark.parametrize("window", [0, 53])
def test_eleven_bits(dsn, D, H, group, page, heads, R, order, lengths, placed, window):
    g = np.random.default_rng(R * D + group + 1)
    pages = Pages(g, lengths, H, D, page)
    idx = [i % len(heads) for i in range(len(lengths))]
    x, got, status = attend(dsn, g, pages, heads, group, idx, R, placed, order, window=window)
    assert status[0] == 0
    check(pages, heads, group, idx, R, placed, x, got, window=window)


@pytest.mark.parametrize("gain", [4.0, 30.0])
@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 1, 4), (64, 5, 5), (128, 60, 1)])
def test_larger_scores(dsn, gain, D, R, group):
    g = np.random.default_rng(17)
    pages = Pages(g, [400, 1000, 160], 2, D, 16)
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 3, R, None, q_gain=gain)
    assert status[0] == 0
    check(pages, [2], group, [0] * 3, R, None, x, got, statistics=False)


@pytest.mark.parametrize("D,R,group,window", [(64, 1, 17, 0), (128, 3, 8, 0), (64, 2, 16, 90), (128, 32, 1, 0), (64, 5, 5, 40), (128, 1, 24, 200)])
def test_items_in_pairs_for_many_requests(dsn, D, R, group, window):
    """17 to 32 query vectors a head, on more requests than CTAs; some of a request's heads and rows, so that pairs and single items alternate."""
    g = np.random.default_rng(R + group)
    lengths = [int(n) for n in g.integers(0, 300, size=230)] + [2500, 640, 33]
    placed = [int(min(n, g.integers(0, R + 1))) for n in lengths]
    placed[-3:] = [R, R, min(R, 33)]
    pages = Pages(g, lengths, 2, D, 32)
    idx = [i % 2 for i in range(len(lengths))]
    x, got, status = attend(dsn, g, pages, [1, 2], group, idx, R, placed, "grouped", window=window)
    assert status[0] == 0
    check(pages, [1, 2], group, idx, R, placed, x, got, window=window)


@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 1, 8), (64, 5, 5), (128, 4, 4), (64, 150, 1), (128, 70, 3)])
@pytest.mark.parametrize("window", [1, 2, 16, 33, 64, 100])
def test_sharp_scores_at_the_edge_of_a_window(dsn, D, R, group, window):
    """Queries that point at the last token they see, at the first, and at the ones beside these two that they do not see."""
    g = np.random.default_rng(window)
    L, B = 331, 4
    pages = Pages(g, [L] * B, 1, D, 16)
    q, target = np.zeros((B, R, 1, group, D)), np.full((B, R, group), -1)
    for i in range(B):
        k, _ = pages.kv(i, 0)
        u = k - k.mean(0)
        for r in range(R):
            me = L - R + r
            for e in range(group):
                t = (me, me - window + 1, me - window, me + 1)[(i + r + e) % 4]
                t = min(max(t, 0), L - 1)
                q[i, r, 0, e] = u[t] / np.linalg.norm(u[t]) * 12
                target[i, r, e] = t
    x, got, status = attend(dsn, g, pages, [1], group, [0] * B, R, None, q=q, scale=4.0, window=window)
    assert status[0] == 0
    check(pages, [1], group, [0] * B, R, None, x, got, scale=4.0, window=window, statistics=False)
    found = 0
    for i in range(B):
        _, v = pages.kv(i, 0)
        for r in range(R):
            me = L - R + r
            for e in range(group):
                t = target[i, r, e]
                off = np.abs(got[i, r, 0, e] - v[t]).max()
                if max(0, me - window + 1) <= t <= me:
                    found += off <= 0.1 * np.abs(v).max()
                else:
                    assert off > 0.1 * np.abs(v).max()            # not what it points at
    assert found
