"""How far attention over the 4-bit cache may be off, from what its two forms round: operands of 11 bits (fp16) behind powers of two, sums in fp32.

U16 = 2^-11 is half a step of fp16 relative to a value, S16 = 2^-25 half its smallest step."""
import numpy as np

from cache_util import U

U16, S16, U32 = 2.0 ** -11, 2.0 ** -25, 2.0 ** -24


def parts(pages, i, head, half):
    """scale (code - 8), middle and scale of the keys (0) or values (1) of request i in a head, [L][D] each."""
    t = np.arange(pages.lengths[i])
    pg, at = pages.table[i, t // pages.page], t % pages.page
    s, z = (np.repeat(a[pg, head, at, half], 64, axis=-1) for a in (pages.s, pages.z))
    code = pages.code[pg, head, at, half].reshape(len(t), pages.D).astype(np.float64)
    return s * (code - 8), z, s


def _movement(scores, e):
    """Scores that are each off by e at most move every weight by a factor within exp(2 e); the exponential and its argument are off by 2^-22 and by U32 of the
    score."""
    e = e + 2.0 ** -22 + 2 * U32 * np.abs(scores)
    return np.expm1(2 * e.max(-1, keepdims=True)) if e.shape[1] else np.zeros((len(e), 1))


def few_rows(pages, i, head, q, p, out, scale):
    """rows * group <= 32.  q [n][D], weights p [n][L], outputs of the formula out [n][D].

    Scores: the query's elements have 8 bits and stay exact behind their power of two, but for those below 2^-13 of the largest, which are off by up to 2^-21 of it
    (every second one is stored as its sixteenth).  Sums start at minus the offsets' product and add numbers up to 1040 |q|: eight roundings of 2^-23 of that,
    times the group's scale.
    Outputs: a probability times a scale is rounded to fp16 (U16 of it; S16 of the unit where it is small, and the unit is below 2^-7 of the largest such product that the row
    sees in the element's group, counting a scale as no less than 2^-50 and a middle's 2^-40th, with a factor of 2 as only exponents are looked at); a middle stays in fp32.
    All sums in fp32: 2^-12 of the terms' sizes."""
    (kc, kz, ks), (vc, vz, vs) = (parts(pages, i, head, half) for half in range(2))
    L, D = kc.shape
    if L == 0 or len(q) == 0:
        return np.full(out.shape, 1e-30)
    k = kc + kz
    top = np.abs(q).max(-1, keepdims=True)
    aq = np.abs(q).reshape(len(q), -1, 64).sum(-1)                                          # [n][groups]
    e = abs(scale) * (8 * 2.0 ** -23 * 1040 * aq @ ks[:, ::64].T + 2.0 ** -21 * top * np.abs(k).sum(-1))
    move = _movement(np.where(p > 0, scale * (q @ k.T), 0.0), np.where(p > 0, e, 0.0))
    size = np.abs(vc) + np.abs(vz)
    unit = np.maximum(np.maximum(vs, np.abs(vz) * 2.0 ** -40), 2.0 ** -50)[:, ::64]         # [L][groups]
    unit = np.repeat((p[:, :, None] * unit[None]).max(1), 64, axis=-1) * 2.0 ** -6
    return U * np.abs(out) + (U16 + 2.0 ** -12 + move) * (p @ size) + L * 8 * S16 * unit + 1e-30


def _greatest_nearby(x):
    """Greatest of x [L] among the 64 tokens that share a tile with each, wherever tiles begin: 63 to either side."""
    pad = np.full(63, -np.inf)
    return np.lib.stride_tricks.sliding_window_view(np.concatenate([pad, x, pad]), 127).max(-1)


def many_rows(pages, i, head, q, p, out, scale, first=0):
    """rows * group > 32: 64 tokens share a power of k and one of v, over all elements and whether a row sees them or not, but for tokens before
    `first`, which stand in front of the windows of all rows.

    Scores: queries as above, S16 of the largest element; a key's element is made in fp16 from its scale and middle, which are exact but for S16 of the tile's greatest,
    and rounded once.  Outputs: the same for values; probabilities are rounded to fp16, S16 of a unit that is up to 2^-7 of the greatest product of a weight
    and a value within a tile."""
    (kc, kz, ks), (vc, vz, vs) = (parts(pages, i, head, half) for half in range(2))
    L, D = kc.shape
    if L == 0 or len(q) == 0:
        return np.full(out.shape, 1e-30)
    k = kc + kz
    counts = np.arange(L) >= first
    near = lambda z, s: 2 * np.maximum(_greatest_nearby(np.where(counts, (np.abs(z) + 8 * s).max(-1), 0.0)), 2.0 ** -50)
    k_near, v_near = near(kz, ks), near(vz, vs)
    top = np.abs(q).max(-1, keepdims=True)
    a = np.abs(q)
    e = abs(scale) * (a @ (U16 * np.abs(k) + 10 * S16 * k_near[:, None]).T + 2 * S16 * top * np.abs(k).sum(-1) + 2.0 ** -18 * a @ np.abs(k).T)
    move = _movement(np.where(p > 0, scale * (q @ k.T), 0.0), np.where(p > 0, e, 0.0))
    size = np.abs(vc) + np.abs(vz)
    p_near = np.stack([_greatest_nearby(row) for row in p])
    unit = (p_near * v_near).max(-1, keepdims=True) * 2.0 ** -7
    return U * np.abs(out) + (2 * U16 + 2.0 ** -12 + move) * (p @ size) + 10 * S16 * (p @ v_near)[:, None] + L * 2 * S16 * unit + 1e-30


# Bounds of every element have to take each rounding at its worst.  What operands are really held in shows in the share of outputs that are not the formula's own
# rounding to bf16: an error e before that rounding changes it with probability e / step.  With operands of 11 bits and weights over tens to thousands of
# tokens that share is 3 to 7 % (few rows: probabilities are rounded) and 5 to 12 % (many rows: keys and values, too); with 8 bits it is eight times the error, 15 to 35 and 35 to
# 59 %.  test_cache_bounds_host.py has both, made from the definition of those roundings.
FEW_SHARE, MANY_SHARE = 0.12, 0.25


def share_off(got, ref):
    from oracle import dsn_oracle as O
    return float(np.mean(got != O.round_bf16(ref)))


def relative(got, ref):
    """Norm of the difference over the norm: 2^-8 / sqrt(3 E[m^2]) for roundings of mantissas m in 1 .. 2 alone, about 2^-9.3."""
    return float(np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()))


RELATIVE = 2.0 ** -9
