"""What the bounds of the 4-bit cache's attention let through, on the host: operands of 11 bits, and nothing that a wrong kernel would give.  No GPU."""
import numpy as np
import pytest

from cache_bounds import FEW_SHARE, MANY_SHARE, RELATIVE, few_rows, many_rows, relative, share_off
from cache_util import Pages
from oracle import dsn_oracle as O


def fp16(x):
    return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def emulated(pages, i, h, q, scale, first, bits, many):
    """The formula with operands rounded where the kernels round them."""
    L, D = pages.lengths[i], pages.D
    t = np.arange(L)
    pg, at = pages.table[i, t // pages.page], t % pages.page
    k, v = pages.kv(i, h)
    s, z = pages.s[pg, h, at, 1], pages.z[pg, h, at, 1]
    code = pages.code[pg, h, at, 1].astype(np.float64) - 8                            # [L][groups][64]
    seen = t <= first + np.arange(len(q))[:, None]
    score = np.where(seen, bits(q) @ (bits(k) if many else k).T * scale, -np.inf)
    p = np.exp(score - score.max(-1, keepdims=True))
    total = p.sum(-1, keepdims=True)
    if many:
        out = bits(p * 128) / 128 @ bits(v)
    else:
        out = np.concatenate([bits(p * s[:, j] * 128) / 128 @ code[:, j] + p @ z[:, j:j + 1] for j in range(D // 64)], -1)
    return O.round_bf16(out / total)


def setting(D, L, n=12, seed=0):
    g = np.random.default_rng(seed + L)
    pages = Pages(g, [L, L], 2, D, 16)
    rows = [(i, h, O.round_bf16(g.normal(size=(n, D)))) for i in range(2) for h in range(2)]
    return pages, rows, D ** -0.5, L - n


def over(pages, rows, scale, first, make, bound):
    """Outputs of `make`: the greatest share of the bound, the share that is not the formula's rounding, the relative norm."""
    got, ref, worst = [], [], 0.0
    for i, h, q in rows:
        k, v = pages.kv(i, h)
        r, p = O.cache_attention(q, k, v, scale, first)
        y = make(i, h, q, k, v, r)
        worst = max(worst, float((np.abs(y - r) / bound(pages, i, h, q, p, r, scale)).max()))
        got.append(y)
        ref.append(r)
    return worst, share_off(np.array(got), np.array(ref)), relative(np.array(got), np.array(ref))


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("D,L", [(64, 30), (64, 300), (64, 2000), (128, 30), (128, 300), (128, 2000)])
def test_eleven_bits_pass_and_eight_do_not(D, L, many):
    pages, rows, scale, first = setting(D, L)
    bound, share = (many_rows, MANY_SHARE) if many else (few_rows, FEW_SHARE)
    worst, off, norm = over(pages, rows, scale, first, lambda i, h, q, *_: emulated(pages, i, h, q, scale, first, fp16, many), bound)
    assert worst <= 1 and off <= share and norm <= RELATIVE
    _, off, norm = over(pages, rows, scale, first, lambda i, h, q, *_: emulated(pages, i, h, q, scale, first, O.round_bf16, many), bound)
    assert off > share
    assert not many or norm > RELATIVE


@pytest.mark.parametrize("bound,share", [(few_rows, FEW_SHARE), (many_rows, MANY_SHARE)])
@pytest.mark.parametrize("D,L", [(64, 30), (64, 300), (64, 2000), (128, 30), (128, 300), (128, 2000)])
def test_wrong_outputs_do_not_pass(D, L, bound, share):
    pages, rows, scale, first = setting(D, L)
    rounded = O.round_bf16
    wrong = {"zeros": lambda i, h, q, k, v, r: np.zeros_like(r),
             "a token more": lambda i, h, q, k, v, r: rounded(O.cache_attention(q, k, v, scale, first + 1)[0]),
             "a token less": lambda i, h, q, k, v, r: rounded(O.cache_attention(q, k, v, scale, first - 1)[0]),
             "without the first": lambda i, h, q, k, v, r: rounded(O.cache_attention(q, k[1:], v[1:], scale, first - 1)[0]),
             "another scale": lambda i, h, q, k, v, r: rounded(O.cache_attention(q, k, v, scale * 1.02, first)[0])}
    for name, make in wrong.items():
        worst, off, norm = over(pages, rows, scale, first, make, bound)
        assert off > share and norm > RELATIVE, name
        if name == "zeros" or L <= 30 and name != "another scale":
            assert worst > 1, name
