"""The residual stream of the norm: written in place while later rows of the same buffer are on their way, alone, and beside codes, in the form that
streams rows through shared memory (for 16 to 256 threads a row) and in the other."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, check_status
from test_gpu_norm_quant import check, code, data, run
from transformer_util import U, groups, half_step, rows_with_pitch, values

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
WIDTHS = [(120, [7, 64, 120]), (384, [384, 190]), (765, [500, 761, 765]), (1000, [1000, 999]), (2048, [1030, 2047, 2048]), (4096, [4095, 2050]),
          (8192, [4100, 8191])]


@pytest.fixture(scope="module")
def ctx(dsn):
    return dsn.Context(0)


def batch(C, k, many):
    g = np.random.default_rng(C + many)
    B = 101 if many else 5
    R = max(15, -(-(5 << 20) // (101 * C)) + 1) if many else 3    # rows enough for the streaming form, or few
    return g, B, R, g.integers(0, len(k), size=B)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("C,k", WIDTHS)
@pytest.mark.parametrize("in_place", ["x", "residual"])
def test_in_place_with_codes(dsn, ctx, name, C, k, in_place):
    g, B, R, idx = batch(C, k, True)
    x, res = data(g, B, R, C, name), data(g, B, R, C, name)
    w = g.uniform(-2, 2, size=C).astype(np.float32).astype(np.float64)
    grouped = C % 1000 == 0
    got = run(dsn, ctx, x, idx, k, name, w, res, in_grouped=grouped, out_grouped=not grouped, in_place=in_place, want_y=C != 384, pitch=16)
    check(got, x, idx, k, name, w, res)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("C,k", WIDTHS)
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("in_place", [None, "x", "residual"])
def test_the_stream_alone(dsn, ctx, name, C, k, many, in_place):
    g, B, R, idx = batch(C, k, many)
    x, res = data(g, B, R, C, name), data(g, B, R, C, name)
    r, perm = groups(dsn, idx, len(k))
    ld = -(-C // 16) * 16
    for grouped in (False, True):
        order = perm if grouped else np.arange(B)
        xd, rd = rows_with_pitch(x[order], ld, DT[name], 7), rows_with_pitch(res[order], ld, DT[name], 9)
        sd = {None: torch.full_like(xd, 11), "x": xd, "residual": rd}[in_place]
        before = values(sd)
        d = dsn.make_norm_desc(code(dsn, name), R, C, k, ldx=ld, ld_res=ld, ld_sum=ld, in_order=int(grouped))
        dsn.dsn_rmsnorm_quant(ctx, d, r, xd, residual=rd, sum_out=sd)
        check_status(ctx, dsn)
        got = values(sd)
        for p, i in enumerate(order):
            c = k[idx[i]]
            h = x[i, :, :c] + res[i, :, :c]
            assert np.all(np.abs(got[p, :, :c] - h) <= (half_step(DT[name]) + U) * np.abs(h))
            np.testing.assert_array_equal(got[p, :, c:], before[p, :, c:])


@pytest.mark.parametrize("many", [False, True])
def test_the_stream_of_a_call_without_residual_is_x(dsn, ctx, many):
    C, k = 384, [384, 190]
    g, B, R, idx = batch(C, k, many)
    x = rows_with_pitch(data(g, B, R, C, "bf16"), C, torch.bfloat16, 0)
    r, _ = groups(dsn, idx, 2)
    sm = torch.full_like(x, 11)
    dsn.dsn_rmsnorm_quant(ctx, dsn.make_norm_desc(dsn.BF16, R, C, k), r, x, sum_out=sm)
    check_status(ctx, dsn)
    for i in range(B):
        c = k[idx[i]]
        assert torch.equal(sm[i, :, :c], x[i, :, :c]) and bool((sm[i, :, c:] == 11).all())
