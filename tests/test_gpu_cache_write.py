"""Keys and values rounded to 4 bits into their pages: codes, pairs and values bit for bit against the definition."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from cache_util import up
from gpu_util import DEV, up_bf16
from transformer_util import groups

pytestmark = pytest.mark.gpu


def place_all(D, page, H, code, s, z, slots, heads_of, pages):
    """Writes rounded rows into host pages; code [B, R, H, 2, n, 64]."""
    n = D // 64
    flat = pages.reshape(-1)
    bits = lambda a: (np.float32(a).view(np.uint32) >> 16).astype(np.uint16)
    for b, r in zip(*np.nonzero(slots >= 0)):
        for h in range(heads_of[b]):
            for half in range(2):
                for grp in range(n):
                    at, _, pair = O.cache_place(D, page, H, int(slots[b, r]), h, half, grp, 0)
                    c = code[b, r, h, half, grp]
                    flat[at:at + 32] = c[0::2] | (c[1::2] << 4)
                    flat[pair:pair + 4] = np.array([bits(s[b, r, h, half, grp]), bits(z[b, r, h, half, grp])], np.uint16).view(np.uint8)


@pytest.mark.parametrize("D,H,group,page,heads,B,R,order", [
    (64, 12, 1, 16, [12], 1, 1, "input"), (64, 5, 1, 64, [1, 3, 5], 9, 13, "grouped"), (64, 5, 3, 48, [2, 5], 7, 6, "input"),
    (128, 4, 2, 16, [4], 3, 50, "grouped"), (128, 3, 16, 1024, [3, 1], 5, 4, "input"), (128, 1, 1, 32, [1], 40, 1, "grouped")])
def test_codes_pairs_and_values(dsn, D, H, group, page, heads, B, R, order):
    g = np.random.default_rng(D + B)
    ctx, T = dsn.Context(0), len(heads)
    idx = g.integers(0, T, size=B)
    r, perm = groups(dsn, idx, T)
    vec = group + 2
    ld, ldv = H * vec * D + 24, H * 2 * D + 8
    x = O.round_bf16(np.exp(g.normal(size=(B, R, H, vec, 1))) * g.normal(size=(B, R, H, vec, D)) + g.normal(size=(B, R, H, vec, 1)))
    x[..., -2, :][g.random(x.shape[:3]) < 0.05] = 3.0                       # constant groups
    x[..., -1, :][g.random(x.shape[:3]) < 0.05] = 0.0
    rows = np.zeros((B, R, ld), np.float32)
    rows[..., :H * vec * D] = x.reshape(B, R, -1)
    n_pages = -(-B * R // page) + 3
    slots = g.permutation(n_pages * page)[:B * R].reshape(B, R)
    slots[g.random((B, R)) < 0.2] = -1
    grouped = order == "grouped"
    lie = perm if grouped else np.arange(B)
    d = dsn.make_cache_desc(R, H, D, heads, group=group, page=page, n_pages=n_pages, order=dsn.GROUPED if grouped else dsn.INPUT_ORDER, ld_qkv=ld,
                            ld_values=ldv)
    assert dsn.dsn_cache_bytes(d) == n_pages * H * (page // 16) * 18 * D
    pages = torch.full((dsn.dsn_cache_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)
    values = torch.full((B, R, ldv), 776.0, dtype=torch.bfloat16, device=DEV)
    c = dsn.make_cache(pages=pages, slots=up(slots))
    qkv = up_bf16(rows[lie])
    kept = qkv.clone()
    dsn.dsn_cache_write_q4(ctx, d, c, r, qkv, values=values)
    assert ctx.get_status()[0] == 0 and torch.equal(qkv, kept)
    code, s, z = O.cache_round(x[..., -2:, :])
    want = np.full(dsn.dsn_cache_bytes(d), 0xA5, np.uint8)
    heads_of = [heads[t] for t in idx]
    place_all(D, page, H, code, s, z, slots, heads_of, want)
    assert np.array_equal(pages.cpu().numpy(), want)
    val = np.full((B, R, ldv), 776.0)
    exact = O.round_bf16(O.cache_values(code, s, z)).reshape(B, R, H, 2 * D)
    for b in range(B):
        for j in range(R):
            if slots[b, j] >= 0:
                val[b, j, :heads_of[b] * 2 * D] = exact[b, j, :heads_of[b]].reshape(-1)
    assert np.array_equal(values.double().cpu().numpy(), val[lie])
    # half a step of the code, what the clamp at the ends cuts off (the middle and the scale are rounded to bf16), and the value's own rounding
    err = np.abs(O.cache_values(code, s, z) - x[..., -2:, :]).reshape(B, R, H, 2, -1, 64).max(-1)
    assert np.all(err <= s * (0.5 + 8 * 2.0 ** -8) + np.abs(z) * 2.0 ** -8 + 1e-30)
    # without values, the same pages; a second write into the same slots replaces the first
    dsn.dsn_cache_write_q4(ctx, d, c, r, -qkv)
    dsn.dsn_cache_write_q4(ctx, d, c, r, qkv)
    assert np.array_equal(pages.cpu().numpy(), want)


@pytest.mark.parametrize("D", [64, 128])
def test_ends_of_the_range(dsn, D):
    ctx = dsn.Context(0)
    big, small = float(O.round_bf16(3.38e38)), 2.0 ** -133
    rows = []
    g = np.random.default_rng(D)
    for lo, hi in ((-big, big), (0.0, big), (-big, -big / 2), (0.0, small), (-small, small), (2.0 ** -126, 2.0 ** -125), (1.0, 1.0 + 2.0 ** -7),
                   (1e-3, 1.01e-3), (-0.0, 0.0)):
        v = O.round_bf16(g.uniform(0, 1, size=2 * D) * (hi / 2 - lo / 2) * 2 + lo)
        v[::5], v[1::5] = O.round_bf16(lo), O.round_bf16(hi)
        rows.append(v)
    x = np.stack(rows).reshape(len(rows), 1, 1, 2, D)
    B = len(rows)
    r, _ = groups(dsn, np.zeros(B, int), 1)
    d = dsn.make_cache_desc(1, 1, D, [1], page=16, n_pages=1, max_pages=1)
    pages = torch.zeros(dsn.dsn_cache_bytes(d), dtype=torch.uint8, device=DEV)
    values = torch.zeros(B, 1, 2 * D, dtype=torch.bfloat16, device=DEV)
    full = np.concatenate([np.zeros((B, 1, 1, 1, D)), x], 3)
    dsn.dsn_cache_write_q4(ctx, d, dsn.make_cache(pages=pages, slots=up(np.arange(B)[:, None])), r, up_bf16(full.reshape(B, 1, -1)), values=values)
    code, s, z = O.cache_round(x)
    want = np.zeros(dsn.dsn_cache_bytes(d), np.uint8)
    place_all(D, 16, 1, code, s, z, np.arange(B)[:, None], [1] * B, want)
    assert np.array_equal(pages.cpu().numpy(), want)
    assert np.all(np.isfinite(values.double().cpu().numpy()))


def test_rows_that_are_not_finite(dsn):
    ctx, D, H = dsn.Context(0), 64, 4
    g = np.random.default_rng(1)
    x = O.round_bf16(g.normal(size=(3, 2, H, 3, D)))
    x[0, 0, 1, 1, 7], x[1, 1, 2, 2, 63], x[2, 0, 0, 2, 0], x[0, 1, 3, 0, 5] = np.nan, np.inf, -np.inf, np.nan   # the last in a query: no matter
    r, _ = groups(dsn, [0, 0, 0], 1)
    d = dsn.make_cache_desc(2, H, D, [H], page=16, n_pages=1)
    pages = torch.zeros(dsn.dsn_cache_bytes(d), dtype=torch.uint8, device=DEV)
    values = torch.zeros(3, 2, H * 2 * D, dtype=torch.bfloat16, device=DEV)
    dsn.dsn_cache_write_q4(ctx, d, dsn.make_cache(pages=pages, slots=up(np.arange(6).reshape(3, 2))), r, up_bf16(x.reshape(3, 2, -1)), values=values)
    got = values.double().cpu().numpy().reshape(3, 2, H, 2, D)
    flat = pages.cpu().numpy()
    for b in range(3):
        for j in range(2):
            for h in range(H):
                poisoned = (b, j, h) in ((0, 0, 1), (1, 1, 2), (2, 0, 0))
                assert np.all(np.isnan(got[b, j, h])) if poisoned else np.all(np.isfinite(got[b, j, h]))
                for half in range(2):
                    _, _, at = O.cache_place(D, 16, H, 2 * b + j, h, half, 0, 0)
                    s, z = (flat[at:at + 4].view(np.uint16).astype(np.uint32) << 16).view(np.float32)
                    assert (s == 0 and np.isnan(z)) if poisoned else np.isfinite(z)


def test_slots_outside_the_cache_are_reported_and_skipped(dsn):
    ctx, D, H, B = dsn.Context(0), 64, 2, 5
    r, _ = groups(dsn, np.zeros(B, int), 1)
    d = dsn.make_cache_desc(1, H, D, [H], page=16, n_pages=2)
    pages = torch.zeros(dsn.dsn_cache_bytes(d) + 64, dtype=torch.uint8, device=DEV)
    x = torch.randn(B, 1, H * 3 * D, device=DEV).to(torch.bfloat16)
    for bad in (32, -2, 2 ** 31 - 1, -2 ** 31):
        pages.zero_()
        slots = up([[3], [bad], [-1], [31], [-1]])
        dsn.dsn_cache_write_q4(ctx, d, dsn.make_cache(pages=pages, slots=slots), r, x)
        assert ctx.get_status() == (dsn.ERR_BAD_INDEX, 1)
        per = 18 * D
        blocks = pages[:-64].view(2, H, 1, per)
        assert all(int((blocks[p, h] != 0).sum()) > 32 for p in range(2) for h in range(H))
        assert int((blocks != 0).sum()) <= 4 * (64 + 8) and int(pages[-64:].sum()) == 0


def test_slots_whose_bytes_lie_beyond_two_to_the_31(dsn):
    ctx, D, H, page = dsn.Context(0), 128, 8, 256
    n_pages = 9000                                              # 9000 * 8 * 16 * 2304 = 2.65e9 bytes
    d = dsn.make_cache_desc(1, H, D, [H], page=page, n_pages=n_pages)
    assert dsn.dsn_cache_bytes(d) > 2 ** 31
    pages = torch.zeros(dsn.dsn_cache_bytes(d), dtype=torch.uint8, device=DEV)
    g = np.random.default_rng(3)
    x = O.round_bf16(g.normal(size=(3, 1, H, 3, D)))
    slots = np.array([[n_pages * page - 1], [5], [8000 * page + 17]])
    r, _ = groups(dsn, [0, 0, 0], 1)
    dsn.dsn_cache_write_q4(ctx, d, dsn.make_cache(pages=pages, slots=up(slots)), r, up_bf16(x.reshape(3, 1, -1)))
    code, s, z = O.cache_round(x[..., 1:, :])
    for b in range(3):
        for h in (0, H - 1):
            at, _, pair = O.cache_place(D, page, H, int(slots[b, 0]), h, 1, 1, 0)
            c = code[b, 0, h, 1, 1]
            assert np.array_equal(pages[at:at + 32].cpu().numpy(), c[0::2] | (c[1::2] << 4))
            assert np.array_equal((pages[pair:pair + 4].cpu().numpy().view(np.uint16).astype(np.uint32) << 16).view(np.float32),
                                  np.array([s[b, 0, h, 1, 1], z[b, 0, h, 1, 1]], np.float32))
