"""Attention over the 4-bit cache against the formula in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from cache_util import Pages, attention_bound, make_desc, up, workspace
from gpu_util import DEV, up_bf16
from transformer_util import groups

pytestmark = pytest.mark.gpu
SENTINEL = 776.0


def attend(dsn, g, pages, heads, group, idx, R, placed, order="input", scale=0.0, window=0, q_gain=1.0, pad=0, q=None):
    """Runs the call; returns queries, outputs [B][R][H][group][D] by request, the context."""
    ctx = dsn.Context(0)
    B, H, D = len(pages.lengths), pages.H, pages.D
    r, perm = groups(dsn, idx, len(heads))
    vec = group + 2
    x = O.round_bf16(g.normal(size=(B, R, H, vec, D)) * q_gain)
    if q is not None:
        x[..., :group, :] = O.round_bf16(q)
    x[..., group:, :] = np.nan                              # this call's k and v are read from the cache alone
    ld, ldo = H * vec * D + pad, H * group * D + pad
    rows = np.zeros((B, R, ld), np.float32)
    rows[..., :H * vec * D] = x.reshape(B, R, -1)
    lie = perm if order == "grouped" else np.arange(B)
    d = make_desc(dsn, pages, R, heads, group, order=dsn.GROUPED if order == "grouped" else dsn.INPUT_ORDER, scale=scale, window=window, ld_qkv=ld, ld_out=ldo)
    c = dsn.make_cache(pages=torch.from_numpy(pages.bytes()).to(DEV), table=up(pages.table), lengths=up(pages.lengths),
                       placed=None if placed is None else up(placed))
    out = torch.full((B, R, ldo), SENTINEL, dtype=torch.bfloat16, device=DEV)
    qkv, ws = up_bf16(rows[lie]), workspace(dsn, d, B)
    dsn.dsn_cache_attention_q4(ctx, d, c, r, qkv, out, ws)
    status = ctx.get_status()
    got = out.double().cpu().numpy()
    back = np.empty_like(got)
    back[lie] = got
    assert np.all(back[..., H * group * D:] == SENTINEL)
    # a second time: the same bits, whatever the workspace holds
    out2 = torch.full_like(out, SENTINEL)
    dsn.dsn_cache_attention_q4(ctx, d, c, r, qkv, out2, ws)
    assert torch.equal(torch.nan_to_num(out.float(), nan=12345.0), torch.nan_to_num(out2.float(), nan=12345.0))
    return x[..., :group, :], back[..., :H * group * D].reshape(B, R, H, group, D), status


def compare(pages, heads, group, idx, R, placed, x, got, scale=0.0, window=0, every=1):
    D = pages.D
    sc = scale or D ** -0.5
    worst = 0.0
    for i, L in enumerate(pages.lengths):
        n = R if placed is None else placed[i]
        assert np.all(got[i, n:] == SENTINEL)               # padding
        assert np.all(got[i, :, heads[idx[i]]:] == SENTINEL)
        if i % every:
            continue
        for h in range(heads[idx[i]]):
            (k, v), size = pages.kv(i, h), pages.v_size(i, h)
            for e in range(group):
                q = x[i, :n, h, e]
                ref, p = O.cache_attention(q, k, v, sc, L - n, window)
                bound = attention_bound(q, k, size, p, ref, sc)
                err = np.abs(got[i, :n, h, e] - ref)
                assert np.all(err <= bound), (i, h, e, float((err / bound).max()))
                if n:
                    worst = max(worst, float((err / bound).max()))
    return worst


CASES = [
    # D, H, group, page, heads, R, order, lengths, placed
    (64, 12, 1, 16, [12], 1, "input", [1], None),
    (64, 3, 1, 16, [1, 3], 1, "grouped", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1023], None),
    (128, 2, 1, 64, [2], 1, "input", [1, 16, 17, 48, 64, 65, 255, 1000], None),
    (128, 2, 4, 16, [1, 2], 1, "grouped", [7, 300, 1, 2000, 33, 0, 128], [1, 1, 1, 1, 1, 0, 1]),
    (64, 2, 8, 48, [2], 1, "input", [5, 49, 777, 2049], None),
    (128, 1, 7, 32, [1], 1, "input", [3, 64, 1025], None),
    (128, 1, 16, 256, [1], 1, "grouped", [300, 31, 2000], None),
    (64, 1, 64, 16, [1], 2, "input", [300, 2, 90], None),
    (128, 2, 16, 16, [1, 2], 2, "grouped", [300, 2, 2000, 31, 65], [2, 2, 1, 2, 0]),   # 32 query vectors a head, or 16, or none
    (64, 3, 17, 32, [3], 1, "input", [1, 64, 129, 5000], None),
    (128, 1, 1, 16, [1], 32, "grouped", [32, 1000, 40], [32, 17, 16]),
    (64, 2, 11, 16, [2], 3, "input", [700, 3], None),                                  # 33
    (64, 4, 2, 32, [2, 4], 5, "grouped", [5, 40, 700, 64, 12], [5, 3, 5, 0, 1]),
    (128, 2, 3, 16, [2], 9, "input", [9, 100, 1000], [9, 9, 2]),
    (128, 1, 1, 1024, [1], 33, "input", [33, 3000, 100], [33, 33, 7]),
    (64, 2, 5, 64, [1, 2], 40, "grouped", [40, 41, 1500, 64], [40, 13, 40, 1]),
    (128, 2, 4, 16, [2], 130, "input", [130, 700, 129, 128], [130, 129, 129, 1]),
    (64, 1, 2, 16, [1], 300, "input", [300, 1200], [300, 257]),
    (128, 1, 1, 48, [1], 257, "grouped", [257, 600], None),
]


@pytest.mark.parametrize("D,H,group,page,heads,R,order,lengths,placed", CASES)
@pytest.mark.parametrize("window", [0, 37])
def test_against_the_formula(dsn, D, H, group, page, heads, R, order, lengths, placed, window):
    g = np.random.default_rng(R * D + group)
    pages = Pages(g, lengths, H, D, page)
    idx = [i % len(heads) for i in range(len(lengths))]
    x, got, status = attend(dsn, g, pages, heads, group, idx, R, placed, order, window=window, pad=8)
    assert status[0] == 0
    compare(pages, heads, group, idx, R, placed, x, got, window=window)


@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 1, 4), (128, 1, 12), (64, 3, 5), (128, 160, 2)])
def test_sharp_scores_find_their_token(dsn, D, R, group):
    """Every query points at one token, whose score stands far above the others: the output is that token's value.  All places at
    which a block, page or tile can end, first and last token included; a token that is not seen yet does not leak."""
    g = np.random.default_rng(D)
    L = 700
    B = 24 if R == 1 else 2
    pages = Pages(g, [L] * B, 1, D, 32)
    edges = sorted({0, 1, L - R} | {e + o for e in (16, 32, 64, 96, 128, 256, 512, 640) for o in (-1, 0, 1) if e + o <= L - R})
    q = np.zeros((B, R, 1, group, D))
    target = np.zeros((B, R, group), int)
    for i in range(B):
        k, _ = pages.kv(i, 0)
        for r in range(R):
            for e in range(group):
                t = edges[(i * R * group + r * group + e) % len(edges)]
                if (r + e) % 3 == 2:
                    t = L - R + r                           # the query's own token
                u = k - k.mean(0)
                q[i, r, 0, e] = u[t] / np.linalg.norm(u[t]) * 12
                target[i, r, e] = t
    x, got, status = attend(dsn, g, pages, [1], group, [0] * B, R, None, q=q, scale=4.0)
    assert status[0] == 0
    compare(pages, [1], group, [0] * B, R, None, x, got, scale=4.0)
    for i in range(B):
        k, v = pages.kv(i, 0)
        for r in range(R):
            for e in range(group):
                _, p = O.cache_attention(x[i, r:r + 1, 0, e], k, v, 4.0, L - R + r)
                if p[0, target[i, r, e]] > 0.999:
                    assert np.max(np.abs(got[i, r, 0, e] - v[target[i, r, e]])) <= 0.05 * np.abs(v).max()


@pytest.mark.parametrize("gain", [1e-30, 1e-3, 30.0, 3e4])
@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 2, 4), (64, 150, 1)])
def test_scores_of_every_size(dsn, gain, D, R, group):
    g = np.random.default_rng(5)
    pages = Pages(g, [400, 1000, 160], 2, D, 16)
    x, got, status = attend(dsn, g, pages, [2], group, [0, 0, 0], R, None, q_gain=gain)
    assert status[0] == 0 and np.all(np.isfinite(got))
    if gain <= 30.0:
        compare(pages, [2], group, [0, 0, 0], R, None, x, got)


@pytest.mark.parametrize("size", ["small", "large", "both", "constant"])
@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 1, 4), (128, 5, 4), (128, 150, 1)])
def test_values_of_every_size(dsn, size, D, R, group):
    """Magnitudes of v from 1e-14 to 1e33.  In "both" the small ones come first, and the large ones show whether their share of the sum is kept."""
    g = np.random.default_rng(15)
    lengths = [3000, 1000, 160]
    pages = Pages(g, lengths, 2, D, 16)
    s, z = pages.s[:, :, :, 1], pages.z[:, :, :, 1]
    gain = np.full(s.shape, {"small": 2.0 ** -44, "large": 2.0 ** 108, "both": 2.0 ** 108, "constant": 1.0}[size])
    for i, L in enumerate(lengths):
        for t in range(L):
            pg, at = pages.table[i, t // 16], t % 16
            if size == "both" and t < L // 128 * 64:              # tokens that share a power are alike
                gain[pg, :, at] = 2.0 ** -44
            if size == "constant" and t % 3 == 0:                # a group of one value has scale 0
                s[pg, :, at], z[pg, :, at] = 0.0, 2.0 ** 100
    s *= gain
    z *= gain
    x, got, status = attend(dsn, g, pages, [2], group, [0, 0, 0], R, None)
    assert status[0] == 0 and np.all(np.isfinite(got))
    compare(pages, [2], group, [0, 0, 0], R, None, x, got)


@pytest.mark.parametrize("scale", [-0.5, 1e-6])
def test_other_scales(dsn, scale):
    g = np.random.default_rng(6)
    pages = Pages(g, [333, 90], 2, 64, 16)
    x, got, _ = attend(dsn, g, pages, [2], 2, [0, 0], 3, None, scale=scale)
    compare(pages, [2], 2, [0, 0], 3, None, x, got, scale=scale)


@pytest.mark.parametrize("D,R,group", [(64, 1, 1), (128, 1, 4), (64, 4, 2), (128, 140, 2)])
def test_tokens_that_are_not_finite_reach_only_the_queries_that_see_them(dsn, D, R, group):
    g = np.random.default_rng(7)
    L = 400
    pages = Pages(g, [L, L, L], 2, D, 32)
    where = [100, L - 1, L - R + R // 2]
    for i, t in enumerate(where):
        pg, at = pages.table[i, t // 32], t % 32
        pages.s[pg, 1, at], pages.z[pg, 1, at], pages.code[pg, 1, at] = 0.0, np.nan, 8
    x, got, status = attend(dsn, g, pages, [2], group, [0, 0, 0], R, None)
    assert status[0] == 0
    for i, t in enumerate(where):
        for r in range(R):
            sees = t <= L - R + r
            assert np.all(np.isnan(got[i, r, 1])) if sees else np.all(np.isfinite(got[i, r, 1]))
            assert np.all(np.isfinite(got[i, r, 0]))
    # what is finite is right: the same queries against a cache whose bad tokens are others, cut off by the window
    for i, t in enumerate(where):
        pg, at = pages.table[i, t // 32], t % 32
        pages.s[pg, 1, at], pages.z[pg, 1, at] = 0.125, 0.5
    for i, t in enumerate(where):
        k, v = pages.kv(i, 1)
        for r in range(R):
            if t > L - R + r:
                for e in range(group):
                    ref, p = O.cache_attention(x[i, r:r + 1, 1, e], k, v, D ** -0.5, L - R + r)
                    assert np.all(np.abs(got[i, r, 1, e] - ref[0]) <= attention_bound(x[i, r:r + 1, 1, e], k, pages.v_size(i, 1), p, ref, D ** -0.5)[0])


@pytest.mark.parametrize("R", [1, 140])
def test_rows_that_see_nothing_are_zero(dsn, R):
    """More rows than tokens: the first of them stand before the request's first token."""
    g = np.random.default_rng(8)
    pages = Pages(g, [0, 3, 200], 2, 64, 16)
    placed = [R, min(R, 7), R]
    x, got, status = attend(dsn, g, pages, [2], 2, [0, 0, 0], R, placed)
    assert status[0] == 0
    assert np.all(got[0] == 0)
    compare(pages, [2], 2, [0, 0, 0], R, placed, x, got)


@pytest.mark.parametrize("R", [1, 140])
def test_pages_and_lengths_outside_the_cache(dsn, R):
    g = np.random.default_rng(9)
    L = 300
    pages = Pages(g, [L, L, L], 1, 64, 16)
    good = pages.table.copy()
    for bad in (-1, pages.n_pages, 2 ** 31 - 1, -2 ** 31):
        pages.table = good.copy()
        pages.table[1, 3] = bad
        x, got, status = attend(dsn, g, pages, [1], 1, [0, 0, 0], R, None)
        assert status == (dsn.ERR_BAD_INDEX, 1)
        pages.table = good
        k, v = pages.kv(1, 0)
        keep = np.r_[0:48, 64:L]                            # that page's tokens are left out
        s = x[1, :, 0, 0] @ k.T / 8
        me = L - R + np.arange(R)[:, None]
        s = np.where((np.arange(L) <= me) & np.isin(np.arange(L), keep), s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        ref = p @ v
        assert np.all(np.abs(got[1, :, 0, 0] - ref) <= attention_bound(x[1, :, 0, 0], k, pages.v_size(1, 0), p, ref, 1 / 8))
    lengths = pages.lengths
    for wrong, used in ((10 ** 9, pages.max_pages * 16), (-5, 0)):
        pages.lengths = [L, wrong, L]
        x, got, status = attend(dsn, g, pages, [1], 1, [0, 0, 0], R, None)
        assert status == (dsn.ERR_BAD_INDEX, 1)
        if used == 0:
            assert np.all(got[1] == 0)
    pages.lengths = lengths
    placed = [R + 1, -3, R]
    x, got, status = attend(dsn, g, pages, [1], 1, [0, 0, 0], R, placed)
    assert status[0] == dsn.ERR_BAD_INDEX and status[1] in (0, 1)
    compare(pages, [1], 1, [0, 0, 0], R, [R, 0, R], x, got)


def test_many_requests(dsn):
    """More requests than threads of a CTA, lengths from nothing to a few pages."""
    g = np.random.default_rng(10)
    B = 1300
    lengths = g.integers(0, 90, size=B)
    lengths[5] = 3000
    pages = Pages(g, lengths.tolist(), 3, 64, 16)
    idx = g.integers(0, 3, size=B)
    placed = [1 if L else 0 for L in lengths]
    x, got, status = attend(dsn, g, pages, [1, 2, 3], 1, idx, 1, placed, "grouped")
    assert status[0] == 0
    compare(pages, [1, 2, 3], 1, idx, 1, placed, x, got)


@pytest.mark.parametrize("R,group", [(1, 1), (1, 8), (200, 4)])
def test_long_request(dsn, R, group):
    g = np.random.default_rng(11)
    L = 20001
    pages = Pages(g, [L, 17 + R], 1, 128, 256)
    x, got, status = attend(dsn, g, pages, [1], group, [0, 0], R, None)
    assert status[0] == 0
    compare(pages, [1], group, [0, 0], R, None, x, got)


@pytest.mark.parametrize("D,group", [(64, 3), (128, 4), (128, 1)])
def test_many_items_one_after_the_other(dsn, D, group):
    """Stretches of many tiles and many items: whole, half filled and cut ones, tiles that only one half of the rows needs."""
    g = np.random.default_rng(13)
    lengths = [int(n) for n in g.integers(1, 400, size=260)] + [4000, 300, 2000, 129]
    R = 90
    placed = [int(min(n, g.integers(0, R + 1))) for n in lengths]
    placed[-4:] = [R, R, 17, R]
    pages = Pages(g, lengths, 2, D, 48)
    idx = [i % 2 for i in range(len(lengths))]
    for window in (0, 70):
        x, got, status = attend(dsn, g, pages, [1, 2], group, idx, R, placed, "grouped", window=window)
        assert status[0] == 0
        compare(pages, [1, 2], group, idx, R, placed, x, got, window=window, every=3)


def test_samples_outside_every_group_are_left_alone(dsn):
    g = np.random.default_rng(12)
    pages = Pages(g, [50, 60, 70], 1, 64, 16)
    ctx = dsn.Context(0)
    r = dsn.make_routing(3, 1, up([2]), up([0, 2]), up([2, 0, -1]), up([1, -1, 0]))
    d = make_desc(dsn, pages, 1, [1], 1)
    c = dsn.make_cache(pages=torch.from_numpy(pages.bytes()).to(DEV), table=up(pages.table), lengths=up(pages.lengths))
    x = torch.randn(3, 1, 192, device=DEV).to(torch.bfloat16)
    out = torch.full((3, 1, 64), SENTINEL, dtype=torch.bfloat16, device=DEV)
    dsn.dsn_cache_attention_q4(ctx, d, c, r, x, out, workspace(dsn, d, 3))
    got = out.double().cpu().numpy()
    assert np.all(got[1] == SENTINEL) and np.all(got[0] != SENTINEL) and np.all(got[2] != SENTINEL)
    q = x.double().cpu().numpy()
    for i in (0, 2):
        k, v = pages.kv(i, 0)
        ref, p = O.cache_attention(q[i, :, :64], k, v, 1 / 8, pages.lengths[i] - 1)
        assert np.all(np.abs(got[i] - ref) <= attention_bound(q[i, :, :64], k, pages.v_size(i, 0), p, ref, 1 / 8))
