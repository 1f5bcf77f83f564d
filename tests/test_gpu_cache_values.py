"""Attention over the 4-bit cache where values differ in size: between the element groups of a head, between tokens that stand side by side, and for tokens that a
row does not see or gives no weight."""
import numpy as np
import pytest

from oracle import dsn_oracle as O
from cache_bounds import few_rows, many_rows
from cache_util import Pages
from test_gpu_cache_attention import attend

pytestmark = pytest.mark.gpu

FEW = [(64, 1, 1), (128, 1, 1), (128, 1, 8), (128, 3, 4), (64, 4, 4), (128, 5, 4), (64, 2, 16)]      # D, rows, queries a head: 1, 8, 12, 16, 20 and 32 vectors
MANY = [(64, 150, 1), (128, 45, 3), (128, 150, 2)]


def put(pages, i, token, groups, gain):
    """The values of a token of request i, in some of its element groups, times gain."""
    pg, at = pages.table[i, token // pages.page], token % pages.page
    pages.s[pg, :, at, 1, groups] *= gain
    pages.z[pg, :, at, 1, groups] *= gain


def check(pages, D, R, group, x, got, bound_of, scale=0.0, window=0):
    sc = scale or D ** -0.5
    for i, L in enumerate(pages.lengths):
        for h in range(pages.H):
            k, v = pages.kv(i, h)
            for e in range(group):
                q = x[i, :, h, e]
                ref, p = O.cache_attention(q, k, v, sc, L - R, window)
                err, bound = np.abs(got[i, :, h, e] - ref), bound_of(pages, i, h, q, p, ref, sc)
                assert np.all(err <= bound), (i, h, e, float((err / bound).max()))


@pytest.mark.parametrize("apart", [22, 34, 60, 110])
@pytest.mark.parametrize("R,group", [(1, 1), (1, 8), (3, 4), (5, 4)])
def test_element_groups_of_different_size(dsn, R, group, apart):
    """The second 64 elements of a head hold values 2^apart below the first, in every other request above."""
    g = np.random.default_rng(apart)
    pages = Pages(g, [3000, 700, 70, 6], 2, 128, 16)
    low = min(apart // 2, 44)
    for i, L in enumerate(pages.lengths):
        for t in range(L):
            put(pages, i, t, i % 2, 2.0 ** (apart - low))
            put(pages, i, t, 1 - i % 2, 2.0 ** -low)
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 4, R, None)
    assert status[0] == 0
    check(pages, 128, R, group, x, got, few_rows)


@pytest.mark.parametrize("D,R,group", FEW)
def test_tokens_side_by_side_of_every_size(dsn, D, R, group):
    """Sizes from 2^-44 to 2^108, drawn for each token and element group."""
    g = np.random.default_rng(D + R)
    pages = Pages(g, [3000, 1000, 160, 20], 2, D, 16)
    for i, L in enumerate(pages.lengths):
        for t in range(L):
            for gr in range(D // 64):
                put(pages, i, t, gr, 2.0 ** int(g.integers(-44, 109)))
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 4, R, None)
    assert status[0] == 0 and np.all(np.isfinite(got))
    check(pages, D, R, group, x, got, few_rows)


@pytest.mark.parametrize("gain", [2.0 ** 22, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("D,R,group", FEW)
def test_large_values_that_no_row_sees(dsn, D, R, group, gain):
    """In front of the window, next to tokens inside it."""
    g = np.random.default_rng(D + R)
    pages = Pages(g, [2000, 300, 70], 2, D, 16)
    window = 37
    for i, L in enumerate(pages.lengths):
        for t in range(L - R - window - 20, L - R - window + 1):      # the first row's window begins one behind the last of them
            if t >= 0:
                put(pages, i, t, slice(None), gain)
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 3, R, None, window=window)
    assert status[0] == 0
    check(pages, D, R, group, x, got, few_rows, window=window)


@pytest.mark.parametrize("gain", [2.0 ** 22, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("D,R,group", [c for c in FEW if c[1] > 1])
def test_large_values_that_only_the_last_row_sees(dsn, D, R, group, gain):
    g = np.random.default_rng(D + R)
    pages = Pages(g, [2000, 300, 70, R], 2, D, 16)
    for i, L in enumerate(pages.lengths):
        put(pages, i, L - 1, slice(None), gain)
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 4, R, None)
    assert status[0] == 0
    check(pages, D, R, group, x, got, few_rows)


@pytest.mark.parametrize("gain", [2.0 ** 22, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("D,R,group", FEW)
def test_large_values_without_weight(dsn, D, R, group, gain):
    """Every query has positive elements, the keys of the large tokens negative ones: their weights are below 2^-100 of the others'."""
    g = np.random.default_rng(D + R)
    pages = Pages(g, [2000, 300, 70], 2, D, 16)
    for i, L in enumerate(pages.lengths):
        for t in sorted({0, L // 3, L // 2, L - R - 9}):
            put(pages, i, t, slice(None), gain)
            pg, at = pages.table[i, t // 16], t % 16
            pages.code[pg, :, at, 0], pages.s[pg, :, at, 0], pages.z[pg, :, at, 0] = 8, 0.25, -4.0
    q = 1.0 + g.random((3, R, 2, group, D))
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 3, R, None, q=q, scale=1.0)
    assert status[0] == 0
    check(pages, D, R, group, x, got, few_rows, scale=1.0)


@pytest.mark.parametrize("apart", [0, 6, 12, 22])
@pytest.mark.parametrize("D,R,group", MANY)
def test_many_rows_hold_what_64_tokens_share(dsn, D, R, group, apart):
    """Sizes up to 2^apart apart, drawn for each token and element group: the bound counts the greatest of 64 tokens in a row, and few bits are lost up to 2^12."""
    g = np.random.default_rng(D + apart)
    pages = Pages(g, [2000, 700, 160], 2, D, 16)
    for i, L in enumerate(pages.lengths):
        for t in range(L):
            for gr in range(D // 64):
                put(pages, i, t, gr, 2.0 ** int(g.integers(0, apart + 1)))
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 3, R, None)
    assert status[0] == 0
    check(pages, D, R, group, x, got, many_rows)


@pytest.mark.parametrize("gain", [2.0 ** 12, 2.0 ** 22, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("D,R,group", [(64, 150, 1), (128, 45, 3), (128, 64, 4), (64, 33, 1)])
def test_many_rows_large_values_in_front_of_every_window(dsn, D, R, group, gain):
    """Up to 256 query vectors: tokens that none of them sees, in the block in which the first row's window begins and in front of it."""
    g = np.random.default_rng(D + R)
    lengths, window = [2000, 700, 161, R + 12], 37
    pages = Pages(g, lengths, 2, D, 16)
    for i, L in enumerate(lengths):
        first = L - R - window + 1
        for t in range(max(0, first - 40), max(0, first)):
            put(pages, i, t, slice(None), gain)
            pg, at = pages.table[i, t // 16], t % 16
            pages.s[pg, :, at, 0] *= gain                             # and their keys
            pages.z[pg, :, at, 0] *= gain
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 4, R, None, window=window)
    assert status[0] == 0
    check(pages, D, R, group, x, got, lambda pg, i, *a: many_rows(pg, i, *a, first=max(0, lengths[i] - R - window + 1)), window=window)


@pytest.mark.parametrize("gain", [2.0 ** 6, 2.0 ** 12])
@pytest.mark.parametrize("D,R,group", MANY)
def test_many_rows_larger_values_that_not_every_row_sees(dsn, D, R, group, gain):
    """The last token of all, tokens in the middle of the rows, and tokens where a window begins."""
    g = np.random.default_rng(D + R)
    pages = Pages(g, [2000, 700, 160], 2, D, 16)
    window = 90
    for i, L in enumerate(pages.lengths):
        for t in {L - 1, L - R // 2, L - R - 1, max(0, L - R - window + 10)}:
            put(pages, i, t, slice(None), gain)
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 3, R, None, window=window)
    assert status[0] == 0
    check(pages, D, R, group, x, got, many_rows, window=window)
