"""Sliced linear layer on 8-bit integers against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV, check_status
from transformer_util import U, groups, half_step, rows_with_pitch, values

pytestmark = pytest.mark.gpu
MARK = 77.0


@pytest.fixture(scope="module")
def ctx(dsn):
    return dsn.Context(0)


def make(seed, B, R, C, N, T, bias=True, bn=False, residual=False):
    g = np.random.default_rng(seed)
    c = dict(idx=g.integers(0, T, size=B), x=g.integers(-127, 128, size=(B, R, C)), W=g.integers(-128, 128, size=(N, C)),
             sx=g.uniform(0.01, 0.05, (B, R)).astype(np.float32).astype(np.float64),
             sw=(g.uniform(0.5, 1.5, N) / 70 / np.sqrt(C)).astype(np.float32).astype(np.float64))
    f = lambda *s: g.normal(size=s).astype(np.float32).astype(np.float64)
    c["bias"] = f(N) if bias else None
    c["bn"] = (1 + 0.2 * f(T, N).astype(np.float32).astype(np.float64), f(T, N)) if bn else None
    if bn:
        c["bn"] = tuple(a.astype(np.float32).astype(np.float64) for a in c["bn"])
    c["res"] = torch.from_numpy(g.normal(size=(B, R, N))).to(torch.bfloat16).double().numpy() if residual else None
    return c


def run(dsn, ctx, c, ki, ko, y="bf16", act=0, in_grouped=False, out_grouped=False, tail=0, pitch=0, call=None):
    B, R, C = c["x"].shape
    N, T = c["W"].shape[0], len(ki)
    r, perm = groups(dsn, c["idx"], T)
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    ldx, ldy = -(-C // 16) * 16 + pitch, -(-N // 8) * 8 + pitch
    xd = rows_with_pitch(c["x"][perm] if in_grouped else c["x"], ldx, torch.int8, 101)   # what lies beyond a slice is not read
    for i, s in enumerate(perm if in_grouped else range(B)):
        xd[i, :, ki[c["idx"][s]]:] = 101
    wd = rows_with_pitch(c["W"][None], ldx, torch.int8, 103)[0]
    f = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)
    sx = f(c["sx"][perm] if in_grouped else c["sx"])
    rd = None if c["res"] is None else rows_with_pitch(c["res"][perm] if out_grouped else c["res"], ldy, dt, float("nan"))
    bn = c["bn"] or (None, None)
    d = dsn.make_linear_i8_desc(R, C, N, ki, ko, wd, f(c["sw"]), bias=f(c["bias"]), bn_scale=f(bn[0]), bn_shift=f(bn[1]), residual=rd,
                                y_dtype=dsn.BF16 if y == "bf16" else dsn.F32, act=act, in_order=int(in_grouped), out_order=int(out_grouped),
                                tail=tail, ldx=ldx, ldw=ldx, ldy=ldy)
    n = dsn.dsn_linear_i8_workspace_bytes(d, B)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    yd = torch.full((B, R, ldy), MARK, dtype=dt, device=DEV)
    (call or dsn.dsn_sliced_linear_i8)(ctx, d, r, xd, sx, yd, ws)
    check_status(ctx, dsn)
    got = values(yd)
    if out_grouped:
        v = np.empty_like(got)
        v[perm] = got
        got = v
    for i in range(B):
        k = ko[c["idx"][i]]
        if tail:
            assert np.all(got[i, :, k:N] == 0)
            k = N
        assert np.all(got[i, :, k:] == MARK)
    return got[..., :N]


def check(got, c, ki, ko, y, act):
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    ref = O.linear_i8(c["x"], c["sx"], c["W"], c["sw"], c["idx"], ki, ko, c["bias"], act, c["bn"], c["res"])
    # fp32 behind an exact sum: its conversion and the factors, the addends: at most 8 roundings of the largest term
    big = np.abs(O.linear_i8(c["x"], c["sx"], c["W"], c["sw"], c["idx"], ki, ko))
    if c["bias"] is not None:
        big = big + np.abs(c["bias"])
    if c["bn"] is not None:
        for i, t in enumerate(c["idx"]):
            big[i] = big[i] * np.abs(c["bn"][0][t]) + np.abs(c["bn"][1][t])
    if c["res"] is not None:
        big = big + np.abs(c["res"])
    tol = 8 * U * big + half_step(dt) * np.abs(ref)
    if act == O.ACT_GELU:
        # slope at most 1.13; the fitted form of bf16 outputs is within 1e-3, erf itself within a few steps of fp32
        tol = 1.13 * tol + (1e-3 if y == "bf16" else 8 * U * big)
    live = ~np.isnan(ref)
    assert np.all(np.abs(got - ref)[live] <= tol[live]), float(np.max((np.abs(got - ref) / tol)[live]))


# few rows in all (a kernel of their own up to 32), one sample in input order, samples tiled alone, many short samples (gathered)
SIZES = [(1, 1, 16, 16), (1, 1, 1, 1), (3, 1, 130, 40), (8, 1, 4096, 100), (9, 1, 65, 33), (1, 17, 1000, 24), (32, 1, 777, 130), (2, 16, 64, 7),
         (33, 1, 512, 64), (5, 9, 96, 70), (40, 7, 200, 300), (3, 64, 129, 130), (3, 65, 300, 257), (2, 197, 384, 520), (1, 300, 100, 260), (7, 128, 48, 9),
         (2500, 2, 40, 24), (700, 9, 200, 100)]


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("B,R,C,N", SIZES)
@pytest.mark.parametrize("in_grouped,out_grouped", [(False, False), (True, True), (True, False), (False, True)])
def test_linear_i8_matches_oracle(dsn, ctx, y, B, R, C, N, in_grouped, out_grouped):
    T = 3
    ki = [max(1, C // 3), max(1, C - 1), C]
    ko = [max(1, N // 2), N, max(1, N - 3)]
    c = make(B * 10 + R + C + N, B, R, C, N, T)
    check(run(dsn, ctx, c, ki, ko, y, 0, in_grouped, out_grouped), c, ki, ko, y, 0)


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("bias,bn,residual", [(False, False, False), (True, True, False), (False, False, True), (True, True, True)])
@pytest.mark.parametrize("B,R", [(7, 3), (11, 40)])
def test_linear_i8_epilogues(dsn, ctx, y, act, bias, bn, residual, B, R):
    C, N, ki, ko = 300, 413, [40, 300], [413, 222]
    c = make(77, B, R, C, N, 2, bias, bn, residual)
    check(run(dsn, ctx, c, ki, ko, y, act, pitch=16), c, ki, ko, y, act)
    check(run(dsn, ctx, c, ki, ko, y, act, in_grouped=True, out_grouped=True, tail=1), c, ki, ko, y, act)


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("act,bias,bn,residual", [(0, True, False, False), (1, False, True, True), (2, True, False, True)])
@pytest.mark.parametrize("B,R,C,N", [(64, 1, 1600, 64), (2, 49, 1100, 61), (1, 197, 4096, 300), (5, 40, 2001, 130), (64, 16, 1030, 600), (33, 1, 16000, 16), (40, 1, 4096, 1024),
                                     (1, 260, 900, 1000)])
def test_linear_i8_long_rows_and_few_tiles(dsn, ctx, y, act, bias, bn, residual, B, R, C, N):
    """Long reductions of tiles fewer than the GPU has room for, paths of one piece beside paths of many, and all samples on one path (more tiles than the
    estimate, which deals samples out evenly)."""
    T = 4
    ki, ko = [100, C, C // 2, C - 1], [N, N // 3, 8, N - 1]
    c = make(B + R + C + N, B, R, C, N, T, bias=bias, bn=bn, residual=residual)
    for grouped in (False, True):
        check(run(dsn, ctx, c, ki, ko, y, act, grouped, not grouped), c, ki, ko, y, act)
    c["idx"][:] = 3
    check(run(dsn, ctx, c, ki, [16, 16, 16, N], y, act, True, True), c, ki, [16, 16, 16, N], y, act)
    c["idx"][:] = 0
    check(run(dsn, ctx, c, ki[:1], [N], y, act, False, True), c, ki[:1], [N], y, act)


def test_linear_i8_extreme_codes_sum_exactly(dsn, ctx):
    """-128 * -128 over the longest rows stays inside 32 bits and is exact; fp32 represents the power of two."""
    C, N = 32752, 64
    for B in (1, 40):
        c = dict(idx=np.zeros(B, int), x=np.full((B, 1, C), -128), W=np.full((N, C), -128), sx=np.full((B, 1), 2.0 ** -20), sw=np.ones(N), bias=None,
                 bn=None, res=None)
        got = run(dsn, ctx, c, [C], [N], "f32")
        np.testing.assert_array_equal(got, 128.0 * 128.0 * C * 2.0 ** -20)


def test_linear_i8_more_slices_than_maps_and_groups_without_samples(dsn, ctx):
    T = 20                                                       # more than 16 distinct slices: two launches
    ki, ko = [20 + 5 * t for t in range(T)], [30 + 7 * t for t in range(T)]
    c = make(3, 50, 5, ki[-1], ko[-1], T)
    c["idx"][c["idx"] % 3 == 0] = 1
    for grouped in (False, True):
        check(run(dsn, ctx, c, ki, ko, "bf16", 0, grouped, grouped), c, ki, ko, "bf16", 0)


def test_linear_i8_many_groups(dsn, ctx):
    g = np.random.default_rng(8)
    B, G, C, N, R = 72, 70, 100, 90, 3
    order = g.permutation(B)
    inv = np.argsort(order)
    slices = np.arange(G) % 2
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)
    r = dsn.make_routing(B, G, up(np.ones(G)), up(np.arange(G + 1)), up(order), up(inv), up(slices))
    c = make(8, B, R, C, N, 2, bias=False)
    idx = np.zeros(B, int)
    idx[order[:G]] = slices
    ki, ko = [64, 100], [90, 33]
    xd = rows_with_pitch(c["x"], 112, torch.int8, 101)
    wd = rows_with_pitch(c["W"][None], 112, torch.int8, 103)[0]
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)
    d = dsn.make_linear_i8_desc(R, C, N, ki, ko, wd, f(c["sw"]), y_dtype=dsn.F32, ldx=112, ldw=112, ldy=92)
    ws = torch.empty(dsn.dsn_linear_i8_workspace_bytes(d, B), dtype=torch.uint8, device=DEV)
    y = torch.full((B, R, 92), MARK, device=DEV)
    dsn.dsn_sliced_linear_i8(ctx, d, r, xd, f(c["sx"]), y, ws)
    check_status(ctx, dsn)
    c["idx"] = idx
    got = values(y)[..., :N]
    assert np.all(got[order[G:]] == MARK)                        # samples that belong to no group
    keep = order[:G]
    sub = {k: (v[keep] if k in ("idx", "x", "sx") else v) for k, v in c.items()}
    check(got[keep], sub, ki, ko, "f32", 0)


def test_linear_i8_workspace_changes_nothing_but_the_time(dsn, ctx):
    c = make(21, 1200, 3, 100, 70, 2)
    seen = []

    def without(ctx_, d, r, x, sx, y, ws):
        seen.append(ws.numel())
        dsn.dsn_sliced_linear_i8(ctx_, d, r, x, sx, y, None)
        a = y.clone()
        y.fill_(MARK)
        dsn.dsn_sliced_linear_i8(ctx_, d, r, x, sx, y, ws[:-16])        # too small: as if there were none
        assert torch.equal(a, y)

    a = run(dsn, ctx, c, [60, 100], [70, 41])
    np.testing.assert_array_equal(run(dsn, ctx, c, [60, 100], [70, 41], call=without), a)
    assert seen == [1200 * 3 * 112]


def test_linear_i8_narrow_rows_on_the_tensor_cores(dsn, ctx):
    """Outputs of a few columns, pitches of 16 bytes, a single input column."""
    for C, N in ((1, 1), (5, 3), (16, 4), (130, 7), (33, 9)):
        for y, ld in (("bf16", -(-N // 8) * 8), ("f32", -(-N // 4) * 4)):
            B = 50
            c = make(C + N, B, 1, C, N, 1)
            dt = torch.bfloat16 if y == "bf16" else torch.float32
            r, _ = groups(dsn, [0] * B, 1)
            f = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)
            ldx = -(-C // 16) * 16
            d = dsn.make_linear_i8_desc(1, C, N, [C], [N], rows_with_pitch(c["W"][None], ldx, torch.int8, 103)[0], f(c["sw"]), bias=f(c["bias"]),
                                        y_dtype=dsn.BF16 if y == "bf16" else dsn.F32, ldx=ldx, ldw=ldx, ldy=ld, in_order=1, out_order=1)
            yd = torch.full((B, 1, ld), MARK, dtype=dt, device=DEV)
            dsn.dsn_sliced_linear_i8(ctx, d, r, rows_with_pitch(c["x"], ldx, torch.int8, 101), f(c["sx"]), yd)
            check_status(ctx, dsn)
            got = values(yd)
            assert np.all(got[..., N:] == MARK)
            check(got[..., :N], c, [C], [N], y, 0)


def test_linear_i8_nan_scales_stay_visible(dsn, ctx):
    for B in (3, 50):
        c = make(5, B, 2, 64, 48, 1)
        c["sx"][1, 0] = np.nan
        for act in (0, 1, 2):
            got = run(dsn, ctx, c, [64], [48], "bf16", act)
            assert np.all(np.isnan(got[1, 0])) and np.isfinite(np.delete(got.reshape(-1, 48), 2, 0)).all()


def test_linear_i8_repeats_bit_for_bit_graph_and_stream(dsn, ctx):
    c = make(6, 20, 100, 256, 300, 2)
    a = run(dsn, ctx, c, [200, 256], [300, 128])

    def on_stream(ctx_, d, r, x, sx, y, ws):
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        dsn.dsn_sliced_linear_i8(ctx_, d, r, x, sx, y, ws, stream=s)
        s.synchronize()

    def captured(ctx_, d, r, x, sx, y, ws):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dsn.dsn_sliced_linear_i8(ctx_, d, r, x, sx, y, ws)
        y.fill_(MARK)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()

    for how in (on_stream, captured):
        np.testing.assert_array_equal(run(dsn, ctx, c, [200, 256], [300, 128], call=how), a)


def test_linear_i8_refusals(dsn, ctx):
    r, _ = groups(dsn, [0, 1], 2)
    x, W = torch.zeros(2, 32, dtype=torch.int8, device=DEV), torch.zeros(48, 32, dtype=torch.int8, device=DEV)
    sx, sw, y = torch.zeros(2, device=DEV), torch.zeros(48, device=DEV), torch.full((2, 48), MARK, dtype=torch.bfloat16, device=DEV)

    def call(code, xx=x, ss=sx, yy=y, ws=None, ki=(16, 32), ko=(48, 8), rr=r, **kw):
        a = dict(R=1, C_in=32, C_out=48, k_in=list(ki), k_out=list(ko), W=W, w_scale=sw)
        a.update(kw)
        with pytest.raises(dsn.DsnError) as e:
            dsn.dsn_sliced_linear_i8(ctx, dsn.make_linear_i8_desc(**a), rr, xx, ss, yy, ws)
        assert e.value.code == code, (e.value.code, kw)

    bad, align = dsn.ERR_INVALID_ARG, dsn.ERR_ALIGNMENT
    call(bad, ki=(0, 32)), call(bad, ki=(16, 33)), call(bad, ko=(49, 8)), call(bad, ki=(16,), ko=(48, 8))
    call(bad, act=3), call(bad, in_order=2), call(bad, tail=2), call(bad, y_dtype=5), call(bad, R=0)
    call(bad, ss=None), call(bad, xx=None), call(bad, yy=None), call(bad, xx=x.to(torch.uint8)), call(bad, ss=sx.bfloat16()), call(bad, yy=y.float())
    call(bad, w_scale=sw[:40]), call(bad, W=W[:40].clone()), call(bad, bias=sw[:40]), call(bad, bn_scale=torch.zeros(96, device=DEV))
    call(bad, residual=y), call(bad, R=2), call(bad, ldx=16)
    call(align, C_out=47, ko=(47, 8)), call(align, C_in=31, ki=(16, 31)), call(align, xx=torch.zeros(96, dtype=torch.int8, device=DEV)[1:])
    call(align, ws=torch.empty(48, dtype=torch.uint8, device=DEV)[1:]), call(bad, ws=torch.empty(48, dtype=torch.uint8))
    torch.cuda.synchronize()
    assert bool((y == MARK).all())
    r0, _ = groups(dsn, [], 2)
    dsn.dsn_sliced_linear_i8(ctx, dsn.make_linear_i8_desc(1, 32, 48, [16, 32], [48, 8], W, sw), r0, x, sx, y)   # an empty batch is fine
