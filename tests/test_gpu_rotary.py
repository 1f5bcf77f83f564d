"""Rotary positions with several axes against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV, check_status
from transformer_util import U, groups, half_step, values

pytestmark = pytest.mark.gpu
MARK = 77.0
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx(dsn):
    return dsn.Context(0)


def run(dsn, ctx, seed, B, N, H, D, heads, pairs, name, vectors=3, rotated=2, per_axis=False, interleaved=False, shared=False, inverse=False,
        grouped=False, in_place=False, pitch=0, offset=0, top=1000, base=10000.0, x=None, pos=None):
    """One call, checked against the oracle; returns (x, y) as the rows lie."""
    g = np.random.default_rng(seed)
    dt = DT[name]
    T = len(heads)
    idx = g.integers(0, T, size=B)
    r, perm = groups(dsn, idx, T)
    rows = idx[perm] if grouped else idx                          # path of every sample as the rows lie
    row = H * vectors * D
    ld = row + pitch
    if pos is None:
        pos = g.integers(-top, top + 1, size=(len(pairs), N if shared else B * N))
    pd = torch.from_numpy(np.ascontiguousarray(pos).astype(np.int32)).to(DEV)
    store = torch.full((B * N * ld + offset,), float("nan"), dtype=dt, device=DEV)
    xd = store[offset:].view(B, N, ld)
    xv = g.normal(size=(B, N, row)) if x is None else x
    xd[..., :row] = torch.from_numpy(xv).to(dt).to(DEV)
    for i in range(B):
        xd[i, :, heads[rows[i]] * vectors * D:row] = float("nan")  # heads that a path does not have are not read
    x0 = values(xd)
    if in_place:
        yd = xd
    else:
        yd = torch.full((B * N * ld + offset,), MARK, dtype=dt, device=DEV)[offset:].view(B, N, ld)
    d = dsn.make_rotary_desc(dsn.BF16 if name == "bf16" else dsn.F32, N, H, D, heads, pairs, vectors=vectors, rotated=rotated, base=base,
                             ladder=int(per_axis), pairing=int(interleaved), shared_positions=shared, inverse=inverse, order=int(grouped),
                             ldx=ld, ldy=ld)
    dsn.dsn_rotary_axes(ctx, d, r, pd, xd, yd)
    check_status(ctx, dsn)
    y = values(yd)
    for i in range(B):
        h = heads[rows[i]]
        live = h * vectors * D
        np.testing.assert_array_equal(y[i, :, live:], x0[i, :, live:] if in_place else np.full_like(y[i, :, live:], MARK))
        v = x0[i, :, :live].reshape(N, h, vectors, D)
        got = y[i, :, :live].reshape(N, h, vectors, D)
        np.testing.assert_array_equal(got[:, :, rotated:], v[:, :, rotated:])
        p = pos[:, :, None, None] if shared else pos[:, i * N:(i + 1) * N, None, None]
        p = np.broadcast_to(p, (len(pairs), N, h, rotated))
        ref = O.rotary_axes(v[:, :, :rotated], p, pairs, base, per_axis, interleaved, inverse)
        P = sum(pairs)
        np.testing.assert_array_equal(got[:, :, :rotated, 2 * P:], v[:, :, :rotated, 2 * P:])
        # the angle: half a step of fp32 of at most one half turn (pi 2^-25) and of its frequency (2^-65 a unit of position); sine and
        # cosine within 2 steps of fp32, two products and a sum: 8 of 2^-24 of |u| + |v|
        a = v[:, :, :rotated, :2 * P]
        mate = np.concatenate([a[..., P:], a[..., :P]], -1) if not interleaved else a.reshape(*a.shape[:-1], P, 2)[..., ::-1].reshape(a.shape)
        tol = 10 * U * (np.abs(a) + np.abs(mate)) + half_step(dt) * np.abs(ref[..., :2 * P])
        err = np.abs(got[:, :, :rotated, :2 * P] - ref[..., :2 * P])
        assert np.all(err <= tol), float(np.max(err / tol))
    return x0, y


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("per_axis", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,N,H,D,heads,pairs", [(1, 1, 1, 2, [1], [1]), (1, 1, 32, 128, [32], [64]), (3, 5, 4, 64, [2, 4], [16, 16]),
                                                 (2, 7, 3, 80, [3], [8, 8, 20]), (5, 3, 2, 34, [1, 2], [5, 7, 5]), (2, 3, 5, 256, [5, 3], [64, 64]),
                                                 (4, 33, 1, 96, [1], [24]), (1, 4, 2, 7, [2], [1, 2])])
def test_rotary_matches_oracle(dsn, ctx, name, per_axis, interleaved, B, N, H, D, heads, pairs):
    kw = dict(per_axis=per_axis, interleaved=interleaved)
    run(dsn, ctx, 1, B, N, H, D, heads, pairs, name, **kw)
    run(dsn, ctx, 2, B, N, H, D, heads, pairs, name, vectors=1, rotated=1, shared=True, grouped=True, in_place=True, **kw)
    run(dsn, ctx, 3, B, N, H, D, heads, pairs, name, vectors=4, rotated=4, inverse=True, pitch=16, **kw)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,D,vectors,heads,pairs", [(3, 16, 3, [1, 3], [8]), (12, 64, 3, [12, 5], [16, 16]), (9, 80, 3, [9], [8, 16, 8]), (32, 128, 2, [32, 31], [64]),
                                                     (24, 256, 4, [24], [8, 40]), (2, 32, 1, [2], [4, 4])])
def test_rotary_of_many_tokens_matches_oracle(dsn, ctx, name, interleaved, H, D, vectors, heads, pairs):
    """Tokens enough for the form that streams rows through shared memory, rows for each number of threads a token."""
    rotated = min(vectors, 2)
    run(dsn, ctx, 11, 41, 31, H, D, heads, pairs, name, vectors=vectors, rotated=rotated, interleaved=interleaved, shared=True)
    run(dsn, ctx, 12, 41, 31, H, D, heads, pairs, name, vectors=vectors, rotated=rotated, interleaved=interleaved, grouped=True, in_place=True,
        per_axis=True, pitch=16, inverse=True)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,D,vectors,heads,pairs", [(6, 7, 8, [3, 6], [1, 2]), (2, 34, 4, [2, 1], [5, 7, 5]), (12, 72, 3, [12, 5], [13, 5]),
                                                     (31, 256, 1, [31, 30], [67]), (24, 256, 4, [24], [8, 41]), (3, 18, 2, [3, 1], [9])])
def test_rotary_of_many_tokens_with_places_that_are_no_16_bytes(dsn, ctx, name, interleaved, H, D, vectors, heads, pairs):
    """Whole rows of 16-byte pieces whose turned halves or vectors begin inside a piece; the last shape has such rows in fp32 alone."""
    rotated = min(vectors, 2)
    run(dsn, ctx, 21, 41, 31, H, D, heads, pairs, name, vectors=vectors, rotated=rotated, interleaved=interleaved, shared=True)
    run(dsn, ctx, 22, 41, 31, H, D, heads, pairs, name, vectors=vectors, rotated=rotated, interleaved=interleaved, grouped=True, in_place=True,
        per_axis=True, pitch=16, inverse=True)


def test_rotary_unaligned_rows_take_the_element_form(dsn, ctx):
    for name in ("bf16", "f32"):
        run(dsn, ctx, 4, 3, 4, 2, 64, [1, 2], [16, 16], name, offset=1)
        run(dsn, ctx, 5, 3, 4, 2, 64, [1, 2], [16, 16], name, pitch=1, in_place=True)


def test_rotary_far_positions_are_exact(dsn, ctx):
    """Angles of positions up to the ends of 32 bits; the double angle of the oracle itself carries 2^31 * 2^-53 of a radian."""
    pos = np.array([[2147483647, -2147483648, 1000000, 16777217, -1, 0, 123456789, 2]])
    run(dsn, ctx, 6, 1, 8, 2, 64, [2], [32], "f32", pos=pos)
    run(dsn, ctx, 6, 1, 8, 2, 64, [2], [32], "f32", pos=pos, base=1.5)


def test_rotary_origin_is_the_identity_and_inverse_is_the_gradient(dsn, ctx):
    x, y = run(dsn, ctx, 7, 2, 6, 2, 64, [2], [16, 16], "bf16", pos=np.zeros((2, 12), int))
    np.testing.assert_array_equal(x, y)
    # <turn(x), w> = <x, turn back(w)> for the formula, and differences of the call along w
    g = np.random.default_rng(8)
    pos = g.integers(0, 50, size=(2, 6))
    w, x = g.normal(size=(1, 6, 128)), g.normal(size=(1, 6, 128))
    kw = dict(vectors=1, rotated=1, pos=pos)
    _, y0 = run(dsn, ctx, 9, 1, 6, 2, 64, [2], [16, 16], "f32", x=x, **kw)
    xg, grad = run(dsn, ctx, 9, 1, 6, 2, 64, [2], [16, 16], "f32", x=w, inverse=True, **kw)
    e = g.normal(size=x.shape)
    _, y1 = run(dsn, ctx, 9, 1, 6, 2, 64, [2], [16, 16], "f32", x=x + e, **kw)
    # 768 products of values below 5, each off by a few steps of fp32: 768 * 25 * 2^-20 at most
    assert abs(np.sum((y1 - y0) * xg) - np.sum(e * grad)) <= 768 * 25 * 2.0 ** -20


def test_rotary_graph_stream_empty_and_many_groups(dsn, ctx):
    r0, _ = groups(dsn, [], 1)
    d = dsn.make_rotary_desc(dsn.F32, 4, 1, 8, [1], [4], vectors=1, rotated=1)
    pos, x = torch.arange(4, dtype=torch.int32, device=DEV), torch.ones(70, 4, 8, device=DEV)
    y = torch.full_like(x, MARK)
    dsn.dsn_rotary_axes(ctx, d, r0, pos, x, y)
    assert bool((y == MARK).all())
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)
    r = dsn.make_routing(70, 66, up(np.ones(66)), up(np.arange(67)), up(np.arange(70)[::-1]), up(np.arange(70)[::-1]), up(np.zeros(66)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsn.dsn_rotary_axes(ctx, d, r, pos, x, y)
    graph.replay()
    torch.cuda.synchronize()
    ref = O.rotary_axes(np.ones((4, 8)), np.arange(4)[None], [4])
    got = values(y)
    assert np.all(got[:4] == MARK) and np.allclose(got[4:], ref, atol=1e-6)
    s = torch.cuda.Stream()
    z = torch.full_like(x, MARK)
    torch.cuda.synchronize()
    dsn.dsn_rotary_axes(ctx, d, r, pos, x, z, stream=s)
    s.synchronize()
    assert torch.equal(y, z)


def test_rotary_refusals(dsn, ctx):
    r, _ = groups(dsn, [0, 0], 1)
    x, y = torch.zeros(2, 3, 48, device=DEV), torch.full((2, 3, 48), MARK, device=DEV)
    pos = torch.zeros(2, 6, dtype=torch.int32, device=DEV)

    def call(code, p=pos, xx=x, yy=y, **kw):
        a = dict(dtype=dsn.F32, N=3, H=2, D=8, heads=[2], pairs=[2, 2], shared_positions=False)
        a.update(kw)
        with pytest.raises(dsn.DsnError) as e:
            dsn.dsn_rotary_axes(ctx, dsn.make_rotary_desc(**a), r, p, xx, yy)
        assert e.value.code == code, (e.value.code, kw)

    bad = dsn.ERR_INVALID_ARG
    call(bad, pairs=[2, 3]), call(bad, pairs=[0, 2]), call(bad, pairs=[-1, 2]), call(bad, heads=[3]), call(bad, heads=[0])
    call(bad, D=1), call(bad, D=257), call(bad, vectors=0), call(bad, rotated=4), call(bad, rotated=0), call(bad, vectors=9)
    call(bad, ladder=2), call(bad, pairing=2), call(bad, base=1.0), call(bad, base=float("nan")), call(bad, base=float("inf")), call(bad, order=2)
    call(bad, ldx=40), call(bad, xx=x.bfloat16()), call(bad, p=pos.long()), call(bad, p=pos[:1]), call(bad, N=4), call(bad, p=None), call(bad, yy=None)
    call(bad, yy=x, ldy=96)
    torch.cuda.synchronize()
    assert bool((y == MARK).all())
