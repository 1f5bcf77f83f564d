"""Attention over the 4-bit cache with queries that are not finite: their own rows come out as NaN, all others as they were."""
import numpy as np
import pytest

from oracle import dsn_oracle as O
from cache_util import Pages
from test_gpu_cache_attention import attend, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("scale", [0.0, -0.25])
@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 1, 4), (64, 3, 5), (128, 5, 4), (64, 40, 1), (128, 150, 2)])
def test_rows_that_are_not_finite(dsn, bad, scale, D, R, group):
    """One element of one query in every request; the keys of the first request have one sign there, so an infinity gives all scores the same one."""
    g = np.random.default_rng(D + R)
    pages = Pages(g, [300, 90, R], 2, D, 16)
    pages.code[:, :, :, 0, 0, 7], pages.code[:, :, :, 0, 0, 8] = 0, 15
    used = np.isfinite(pages.s[:, :, :, 0, 0])
    pages.z[:, :, :, 0, 0] = np.where(used, np.clip(pages.z[:, :, :, 0, 0], -0.5, 0.5), np.nan)      # code 0 is below zero, code 15 above
    q = O.round_bf16(g.normal(size=(3, R, 2, group, D)))
    clean = q.copy()
    where = [(0, R // 2, 1, group - 1, 7), (0, 0, 0, 0, 8), (1, R - 1, 0, 0, 8), (2, 0, 1, 0, 7)]
    for i, r, h, e, d in where:
        q[i, r, h, e, d] = bad
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 3, R, None, q=q, scale=scale)
    assert status[0] == 0
    for i, r, h, e, d in where:
        assert np.all(np.isnan(got[i, r, h, e])), (i, r, h, e)
    # the others: as with a finite query there
    x, whole, _ = attend(dsn, g, pages, [2], group, [0] * 3, R, None, q=clean, scale=scale)
    compare(pages, [2], group, [0] * 3, R, None, x, whole, scale=scale)
    touched = np.zeros(got.shape[:4], bool)
    for i, r, h, e, d in where:
        touched[i, r, h, e] = True
    assert np.all(np.isfinite(got[~touched]))
    if R * group > 32:
        assert np.array_equal(got[~touched], whole[~touched])


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("D,R,group", [(64, 8, 1), (128, 7, 4), (64, 60, 1), (128, 150, 2)])
def test_rows_that_see_nothing_are_zero_whatever_they_hold(dsn, bad, D, R, group):
    """Rows in front of a request's first token, some beside rows that see tokens."""
    g = np.random.default_rng(D + R)
    lengths = [0, 1, R - 2, 3]
    pages = Pages(g, lengths, 2, D, 16)
    q = O.round_bf16(g.normal(size=(4, R, 2, group, D)))
    for i, L in enumerate(lengths):
        q[i, :R - L, :, :, ::3] = bad
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 4, R, None, q=q)
    assert status[0] == 0
    for i, L in enumerate(lengths):
        assert np.all(got[i, :R - L] == 0)
        q[i, :R - L] = 0.0
    compare(pages, [2], group, [0] * 4, R, None, q, got)
