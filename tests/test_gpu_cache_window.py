"""Attention over the 4-bit cache with windows up to the type's end and rows in front of a request's first token."""
import numpy as np
import pytest

from cache_util import Pages
from test_gpu_cache_attention import attend, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,R,group", [(64, 8, 1), (128, 3, 4), (64, 5, 6), (128, 8, 4), (64, 40, 1), (128, 150, 2)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2 ** 24, 2 ** 30, -1, 0, 1, 4])
def test_long_windows_hide_nothing(dsn, D, R, group, window):
    """Small numbers are counted from the most tokens that a request can hold, where a window begins to hide nothing."""
    g = np.random.default_rng(D + R)
    pages = Pages(g, [5, 0, 3, 200, 1], 2, D, 16)
    if window < 8:
        window += pages.max_pages * pages.page
    x, got, status = attend(dsn, g, pages, [1, 2], group, [0, 1, 1, 0, 1], R, None, "grouped", window=window)
    assert status[0] == 0
    assert np.all(got[1] == 0)                       # a request without tokens, whose path has both heads
    compare(pages, [1, 2], group, [0, 1, 1, 0, 1], R, None, x, got, window=window)


@pytest.mark.parametrize("D,R,group", [(64, 8, 1), (128, 8, 4), (128, 150, 2)])
@pytest.mark.parametrize("window", [1, 2, 7])
def test_short_windows_in_front_of_the_first_token(dsn, D, R, group, window):
    g = np.random.default_rng(D + R)
    pages = Pages(g, [5, 3, 200, 1], 2, D, 16)
    x, got, status = attend(dsn, g, pages, [2], group, [0] * 4, R, None, window=window)
    assert status[0] == 0
    compare(pages, [2], group, [0] * 4, R, None, x, got, window=window)
