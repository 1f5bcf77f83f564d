"""The 4-bit cache with more than 32 paths, whose groups are searched another way."""
import numpy as np
import pytest

from cache_util import Pages
from test_gpu_cache_accuracy import check
from test_gpu_cache_attention import attend
from test_gpu_cache_write import test_codes_pairs_and_values as write_everything

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,R,group,T", [(64, 1, 1, 33), (128, 1, 4, 64), (64, 9, 2, 40), (64, 45, 1, 64)])
@pytest.mark.parametrize("order", ["input", "grouped"])
def test_attention(dsn, D, R, group, T, order):
    g = np.random.default_rng(T)
    lengths = [int(n) for n in g.integers(0, 120, size=90)]
    pages = Pages(g, lengths, 3, D, 16)
    heads, idx = [1 + t % 3 for t in range(T)], [int(t) for t in g.integers(0, T, size=90)]
    x, got, status = attend(dsn, g, pages, heads, group, idx, R, None, order)
    assert status[0] == 0
    check(pages, heads, group, idx, R, None, x, got, statistics=False)


@pytest.mark.parametrize("order", ["input", "grouped"])
def test_write(dsn, order):
    write_everything(dsn, 64, 3, 1, 16, [1 + t % 3 for t in range(50)], 70, 3, order)
