"""Residual + root-mean-square norm + 8-bit codes against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV, check_status
from transformer_util import U, groups, half_step, rows_with_pitch, values

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
MARK = 77.0


@pytest.fixture(scope="module")
def ctx(dsn):
    return dsn.Context(0)


def code(dsn, name):
    return dsn.BF16 if name == "bf16" else dsn.F32


def run(dsn, ctx, x, idx, k, name, weight=None, residual=None, eps=1e-6, in_grouped=False, out_grouped=False, raw=False, want_y=True,
        in_place=None, pitch=0, stream=None):
    """Returns what the call wrote, in input order: sum, q, scale, y (numpy), and the untouched columns' check is made here."""
    B, R, C = x.shape
    T = len(k)
    r, perm = groups(dsn, idx, T)
    dt = DT[name]
    ld = -(-C // 16) * 16 + pitch
    src = x[perm] if in_grouped else x
    xd = rows_with_pitch(src, ld, dt, 1e30)                     # what lies beyond a slice is neither read nor written
    kept = [k[idx[i]] for i in (perm if in_grouped else range(B))]
    for i, c in enumerate(kept):
        xd[i, :, c:] = 1e30
    rd = None
    if residual is not None:
        rd = rows_with_pitch(residual[perm] if in_grouped else residual, ld, dt, float("nan"))
        for i, c in enumerate(kept):
            rd[i, :, c:] = float("nan")
    sd = {None: torch.full_like(xd, MARK), "x": xd, "residual": rd}[in_place]
    q = None if raw else torch.full((B, R, ld), 99, dtype=torch.int8, device=DEV)
    sc = None if raw else torch.full((B, R), MARK, device=DEV)
    y = torch.full((B, R, ld), MARK, dtype=dt, device=DEV) if want_y or raw else None
    wd = None if weight is None else torch.from_numpy(weight.astype(np.float32)).to(DEV)
    d = dsn.make_norm_desc(code(dsn, name), R, C, k, wd, eps=eps, ldx=ld, ld_res=ld, ld_sum=ld, ldq=ld, ldy=ld,
                           in_order=int(in_grouped), out_order=int(out_grouped))
    before = sd.clone()
    dsn.dsn_rmsnorm_quant(ctx, d, r, xd, q=q, scale=sc, y=y, residual=rd, sum_out=sd, stream=stream)
    check_status(ctx, dsn)
    out = []
    for t, grouped, fill in ((sd, in_grouped, before), (q, out_grouped, 99), (sc, out_grouped, None), (y, out_grouped, MARK)):
        if t is None:
            out.append(None)
            continue
        v = values(t)
        if grouped:
            w = np.empty_like(v)
            w[perm] = v
            v = w
        if fill is not None:
            f = fill
            if isinstance(fill, torch.Tensor):
                f = values(fill)
                if grouped:
                    w = np.empty_like(f)
                    w[perm] = f
                    f = w
            for i in range(B):
                c = k[idx[i]]
                want = f[i, :, c:] if isinstance(f, np.ndarray) else np.full_like(v[i, :, c:], f)
                np.testing.assert_array_equal(v[i, :, c:], want)
        out.append(v)
    return out


def check(got, x, idx, k, name, weight, residual, eps=1e-6):
    sm, q, sc, y = got
    dt = DT[name]
    hs = half_step(dt)
    h, n, scale, steps = O.rmsnorm_quant(x, idx, k, weight, eps, residual)
    for i in range(x.shape[0]):
        c = k[idx[i]]
        # h: one fp32 addition (exact for bf16 halves of like size), one rounding to the stream's type
        assert np.all(np.abs(sm[i, :, :c] - h[i, :, :c]) <= (hs + U) * np.abs(h[i, :, :c]) + 1e-37)
        if q is not None:
            # h w: the sum's and the product's rounding, 127 / max: the maximum's two and its own, one more product: 6 of 2^-24 of at most 127
            assert np.all(np.abs(q[i, :, :c] - steps[i, :, :c]) <= 0.5 + 127 * 7 * U)
            # the sum of c squares: a thread adds at most 32, then 5 shuffles and at most 32 partial sums: 70 roundings at most, halved by the root
            assert np.all(np.abs(sc[i] - scale[i]) <= 48 * U * scale[i])
            if y is not None:
                ref = q[i, :, :c] * sc[i][:, None]
                assert np.all(np.abs(y[i, :, :c] - ref) <= (hs + 2 * U) * np.abs(ref))
        else:
            assert np.all(np.abs(y[i, :, :c] - n[i, :, :c]) <= (hs + 48 * U) * np.abs(n[i, :, :c]) + 1e-37)


def data(g, B, R, C, name):
    size = np.exp(0.7 * g.normal(size=C))
    x = g.normal(size=(B, R, C)) * size
    return torch.from_numpy(x).to(DT[name]).double().numpy()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("B,R,C,k", [(1, 1, 8, [8]), (1, 1, 768, [768]), (3, 1, 1, [1]), (5, 3, 7, [3, 7]), (6, 5, 100, [1, 33, 100]),
                                     (4, 7, 257, [256, 257]), (7, 2, 513, [64, 512, 513]), (3, 5, 1000, [511, 1000]), (2, 3, 1030, [1025, 1030]),
                                     (2, 2, 2049, [2048, 2049]), (3, 2, 4097, [4096, 4097]), (2, 2, 9000, [8192, 9000]), (1, 2, 20001, [20001])])
def test_norm_matches_oracle(dsn, ctx, name, B, R, C, k):
    g = np.random.default_rng(B * 100 + C)
    idx = g.integers(0, len(k), size=B)
    x, res = data(g, B, R, C, name), data(g, B, R, C, name)
    w = g.uniform(-2, 2, size=C).astype(np.float32).astype(np.float64)
    check(run(dsn, ctx, x, idx, k, name, w, res), x, idx, k, name, w, res)
    check(run(dsn, ctx, x, idx, k, name, None, None, raw=True), x, idx, k, name, None, None)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("C,k", [(120, [7, 64, 120]), (250, [130, 250]), (384, [384, 190]), (765, [500, 761, 765]), (1000, [1000, 999]), (2048, [1030, 2047, 2048]),
                                 (4096, [4095, 2050]), (8192, [4100, 8191])])
def test_norm_of_many_rows_matches_oracle(dsn, ctx, name, C, k):
    """Rows enough for the form that streams them through shared memory, one width list for each number of threads a row."""
    g = np.random.default_rng(C)
    B, R = 101, max(15, -(-(5 << 20) // (101 * C)) + 1)
    idx = g.integers(0, len(k), size=B)
    x, res = data(g, B, R, C, name), data(g, B, R, C, name)
    w = g.uniform(-2, 2, size=C).astype(np.float32).astype(np.float64)
    check(run(dsn, ctx, x, idx, k, name, w, res, out_grouped=True), x, idx, k, name, w, res)
    check(run(dsn, ctx, x, idx, k, name, w, None, in_grouped=True, raw=C == 384), x, idx, k, name, w, None)


def test_many_rows_with_tight_last_row_bad_rows_and_large_rows(dsn, ctx):
    """The last row ends with the tensor; rows that are no numbers and rows whose squares overflow stand among ordinary ones."""
    g = np.random.default_rng(12)
    for C, B in ((77, 1300), (77, 70000), (1501, 1300), (1501, 4000)):   # either form
        R, ld = 1, -(-C // 16) * 16
        x = g.normal(size=(B, R, C)).astype(np.float32).astype(np.float64)
        x[5, 0, C - 1], x[17, 0, 3], x[B - 1, 0, 0] = np.nan, np.inf, 3.0
        x[6] *= 2.0 ** 70
        x[7] *= 2.0 ** -125
        x[8] = 0
        store = torch.empty((B - 1) * ld + C, device=DEV)
        xd = store.as_strided((B, C), (ld, 1))
        xd.copy_(torch.from_numpy(x[:, 0].astype(np.float32)))
        r, _ = groups(dsn, [0] * B, 1)
        q, sc = torch.zeros(B, ld, dtype=torch.int8, device=DEV), torch.zeros(B, device=DEV)
        y = torch.zeros(B, ld, device=DEV)
        d = dsn.make_norm_desc(dsn.F32, R, C, [C], eps=1e-20, ldx=ld, ldq=ld, ldy=ld)
        dsn.dsn_rmsnorm_quant(ctx, d, r, xd, q=q, scale=sc, y=y)
        check_status(ctx, dsn)
        got, s, v = values(q)[:, :C], values(sc), values(y)[:, :C]
        for i in (5, 17):
            assert np.isnan(s[i]) and np.all(got[i] == 0) and np.all(np.isnan(v[i]))
            x[i] = 0
        h, n, scale, steps = O.rmsnorm_quant(x, [0] * B, [C], None, 1e-20)
        keep = [i for i in range(B) if i not in (5, 17)]
        assert np.all(np.abs(got[keep] - steps[keep, 0]) <= 0.5 + 127 * 7 * U)
        keep.remove(7)                                            # its squares are below fp32's smallest; the code is exact, the scale is eps's
        np.testing.assert_allclose(s[keep], scale[keep, 0], rtol=48 * U)


@pytest.mark.parametrize("in_grouped", [False, True])
@pytest.mark.parametrize("out_grouped", [False, True])
@pytest.mark.parametrize("in_place", [None, "x", "residual"])
def test_norm_orders_in_place_and_pitch(dsn, ctx, in_grouped, out_grouped, in_place):
    g = np.random.default_rng(9)
    B, R, C, k = 23, 9, 200, [33, 96, 150, 200]
    idx = g.integers(0, 3, size=B)                                # the last path has no sample
    x, res = data(g, B, R, C, "bf16"), data(g, B, R, C, "bf16")
    w = g.uniform(0.5, 2, size=C).astype(np.float32).astype(np.float64)
    got = run(dsn, ctx, x, idx, k, "bf16", w, res, in_grouped=in_grouped, out_grouped=out_grouped, in_place=in_place, pitch=48)
    check(got, x, idx, k, "bf16", w, res)


def test_codes_are_the_same_for_any_scale_of_the_row_and_ties_go_to_even(dsn, ctx):
    # row: 127 * 2^e at the top, so that a code is the value itself over 2^e; halves round to even
    vals = np.array([127, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 63.5, 64.5, 0, -127, 126.5, -126.5, 1, 3.5, 4.5])
    want = np.array([127, 0, 2, 2, 0, -2, -2, 64, 64, 0, -127, 126, -126, 1, 4, 4])
    x = np.stack([vals * 2.0 ** e for e in (-130, -100, -20, 0, 20, 100, 120)])[None]
    got = run(dsn, ctx, x, [0], [16], "f32", eps=1e-20)
    for e in range(x.shape[1]):
        if e > 0:                                                 # 2^-130: the half steps are below fp32's smallest steps only for e < -149
            np.testing.assert_array_equal(got[1][0, e, :16], want)
    np.testing.assert_array_equal(got[1][0, 0, :16], want)
    ref = O.rmsnorm_quant(x, [0], [16], None, 1e-20)
    for e in range(2, x.shape[1]):                                # below, eps dominates; squares beyond fp32 are scaled first
        np.testing.assert_allclose(got[2][0, e], ref[2][0, e], rtol=48 * U)


def test_zero_rows_and_rows_that_are_no_numbers(dsn, ctx):
    g = np.random.default_rng(4)
    x = g.normal(size=(2, 6, 300))
    x[0, 1] = 0
    x[0, 3, 17] = np.nan
    x[1, 0, 299] = np.inf
    x[1, 2, 0] = -np.inf
    for name in ("bf16", "f32"):
        for raw in (False, True):
            xr = torch.from_numpy(x).to(DT[name]).double().numpy()
            sm, q, sc, y = run(dsn, ctx, xr, [0, 0], [300], name, raw=raw)
            bad = np.zeros((2, 6), bool)
            bad[0, 3] = bad[1, 0] = bad[1, 2] = True
            assert np.all(np.isnan(y[bad][:, :300])) and np.all(np.isfinite(y[~bad][:, :300]))
            assert np.all(y[0, 1, :300] == 0)
            if not raw:
                assert np.all(np.isnan(sc[bad])) and np.all(q[bad][:, :300] == 0) and sc[0, 1] == 0 and np.all(q[0, 1, :300] == 0)
            good = [(0, r) for r in (0, 2, 4, 5)] + [(1, r) for r in (1, 3, 4, 5)]
            ref = O.rmsnorm_quant(np.nan_to_num(xr, posinf=0, neginf=0), [0, 0], [300])
            for i, r in good:
                assert np.all(np.abs(y[i, r, :300] - (ref[1][i, r] if raw else q[i, r, :300] * ref[2][i, r])) <= (half_step(DT[name]) + 60 * U) * np.abs(y[i, r, :300]) + 1e-30)


def test_empty_batch_many_groups_and_unrouted_samples(dsn, ctx):
    g = np.random.default_rng(5)
    r, _ = groups(dsn, [], 2)
    d = dsn.make_norm_desc(dsn.F32, 4, 16, [8, 16])
    t = torch.ones(1, 16, device=DEV)
    y = torch.full((1, 16), MARK, device=DEV)
    dsn.dsn_rmsnorm_quant(ctx, d, r, t, y=y)
    assert bool((y == MARK).all())
    # 70 groups of one sample (binary search instead of one load per lane), slices shared by several groups; the last two positions
    # belong to no group
    B, G, C, k = 72, 70, 24, [5, 24, 16]
    order = g.permutation(B).astype(np.int32)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)
    inv = np.empty(B, np.int32)
    inv[order] = np.arange(B)
    slices = np.arange(G) % 3
    rt = dsn.make_routing(B, G, up(np.ones(G)), up(np.arange(G + 1)), up(order), up(inv), up(slices))
    x = g.normal(size=(B, 2, C)).astype(np.float32)
    xd, y = torch.from_numpy(x).to(DEV), torch.full((B, 2, C), MARK, device=DEV)
    dsn.dsn_rmsnorm_quant(ctx, dsn.make_norm_desc(dsn.F32, 2, C, k), rt, xd, y=y)
    check_status(ctx, dsn)
    got = values(y)
    for p in range(B):
        i = order[p]
        c = k[slices[p]] if p < G else 0
        if c:
            n = O.rmsnorm_quant(x[i:i + 1].astype(np.float64), [0], [c])[1]
            np.testing.assert_allclose(got[i, :, :c], n[0, :, :c], rtol=60 * U)
        assert np.all(got[i, :, c:] == MARK)


def test_norm_graph_and_other_stream(dsn, ctx):
    g = np.random.default_rng(6)
    B, R, C = 4, 30, 384
    x = torch.from_numpy(g.normal(size=(B, R, C))).to(torch.bfloat16).to(DEV)
    r, _ = groups(dsn, [0] * B, 1)
    d = dsn.make_norm_desc(dsn.BF16, R, C, [C])
    q, sc, y = (torch.zeros(B, R, C, dtype=t, device=DEV) for t in (torch.int8, torch.float32, torch.bfloat16))
    sc = sc[..., 0].contiguous()
    dsn.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=sc, y=y)
    want = [t.clone() for t in (q, sc, y)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for t in (q, sc, y):
        t.zero_()
    torch.cuda.synchronize()
    dsn.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=sc, y=y, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((q, sc, y), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsn.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=sc, y=y)
    x.mul_(2)                                                     # same codes, scales nearly unchanged (eps)
    q.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, want[0])


def test_norm_refusals(dsn, ctx):
    x = torch.zeros(4, 32, device=DEV)
    q, sc, y = torch.zeros(4, 32, dtype=torch.int8, device=DEV), torch.zeros(4, device=DEV), torch.full((4, 32), MARK, device=DEV)
    r, _ = groups(dsn, [0, 1, 0, 1], 2)

    def call(code, k=(16, 32), dt=None, xx=x, **kw):
        args = dict(q=q, scale=sc, y=y)
        desc = {n: kw.pop(n) for n in list(kw) if n in ("eps", "ldx", "ldq", "ldy", "ld_res", "ld_sum", "in_order", "out_order", "R", "Cn", "weight")}
        args.update(kw)
        with pytest.raises(dsn.DsnError) as e:
            dsn.dsn_rmsnorm_quant(ctx, dsn.make_norm_desc(dsn.F32 if dt is None else dt, desc.pop("R", 1), desc.pop("Cn", 32), list(k), **desc),
                                  r, xx, **args)
        assert e.value.code == code, (e.value.code, kw)

    bad, align = dsn.ERR_INVALID_ARG, dsn.ERR_ALIGNMENT
    call(bad, scale=None)
    call(bad, q=None)
    call(bad, q=None, scale=None, y=None)
    call(bad, k=(0, 32)), call(bad, k=(16, 33)), call(bad, k=(16,))
    call(bad, eps=0.0), call(bad, eps=float("nan")), call(bad, eps=float("inf"))
    call(bad, ldx=16), call(align, ldx=33, xx=torch.zeros(8, 32, device=DEV)), call(align, ldq=40, q=torch.zeros(8, 32, dtype=torch.int8, device=DEV))
    call(bad, in_order=2), call(bad, out_order=-1), call(bad, R=0), call(bad, dt=7)
    call(bad, y=x), call(bad, sum_out=y), call(bad, R=2)          # the last: too few elements for two rows a sample
    call(bad, xx=x.cpu()), call(bad, xx=x.bfloat16())
    call(bad, xx=x, sum_out=x, ld_sum=64)
    call(align, xx=torch.zeros(200, device=DEV)[1:])
    call(align, weight=torch.zeros(40, device=DEV)[1:])
    torch.cuda.synchronize()
    assert bool((y == MARK).all())
