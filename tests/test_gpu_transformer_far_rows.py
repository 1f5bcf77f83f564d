"""The 8-bit transformer operators on buffers of more than 2^31 elements: the rows at the end come out as they do alone."""
import pytest
import torch

from gpu_util import DEV, check_status
from transformer_util import U, groups

pytestmark = pytest.mark.gpu
LAST = 200                                                        # rows compared


def need(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB")


def pattern(rows, cols, dtype, scale=3.0):
    """Values that differ from row to row, made in place, a block of rows at a time."""
    t = torch.empty(rows, cols, dtype=dtype, device=DEV)
    c = torch.arange(cols, device=DEV) * 0.37
    for r0 in range(0, rows, 1 << 14):
        r = torch.arange(r0, min(rows, r0 + (1 << 14)), device=DEV)
        t[r0:r0 + (1 << 14)] = (torch.sin(r[:, None] * 0.71 + c) * scale).to(dtype)
    return t


@pytest.fixture(autouse=True)
def release():
    yield
    torch.cuda.empty_cache()


def test_norm_far_rows(dsn):
    need(24)
    ctx = dsn.Context(0)
    C = 4096
    rows = (1 << 31) // C + 1000
    x, res = pattern(rows, C, torch.bfloat16), pattern(rows, C, torch.bfloat16, 2.0)
    tail = x[-LAST:].clone(), res[-LAST:].clone()

    def call(x, res):
        n = x.shape[0]
        r, _ = groups(dsn, [0], 1)
        q, sc, y = torch.zeros(n, C, dtype=torch.int8, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, C, dtype=torch.bfloat16, device=DEV)
        dsn.dsn_rmsnorm_quant(ctx, dsn.make_norm_desc(dsn.BF16, n, C, [C]), r, x, q=q, scale=sc, y=y, residual=res, sum_out=x)
        check_status(ctx, dsn)
        return x[-LAST:], q[-LAST:], sc[-LAST:], y[-LAST:]

    far, near = call(x, res), call(*tail)
    assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
    # the sum of squares in another order: as in the test against 64 bits; y is a code times its scale
    assert bool(((far[2] - near[2]).abs() <= 2 * 48 * U * near[2]).all())
    assert bool(((far[3].float() - near[3].float()).abs() <= 2.0 ** -7 * near[3].float().abs()).all())


@pytest.mark.parametrize("wide_in", [True, False])
def test_linear_far_rows(dsn, wide_in):
    need(16)
    ctx = dsn.Context(0)
    C, N = (4096, 64) if wide_in else (64, 4096)
    rows = (1 << 31) // 4096 + 1000
    x = pattern(rows, C, torch.float32, 120.0).to(torch.int8) if not wide_in else pattern(rows, C, torch.bfloat16, 120.0).to(torch.int8)
    W = pattern(N, C, torch.float32, 120.0).to(torch.int8)
    sx, sw = torch.linspace(0.01, 0.02, rows, device=DEV), torch.linspace(1e-3, 2e-3, N, device=DEV)

    def call(x, sx, samples):
        n = x.shape[0]
        r, _ = groups(dsn, [0] * samples, 1)
        d = dsn.make_linear_i8_desc(n // samples, C, N, [C], [N], W, sw, in_order=dsn.GROUPED if samples == 1 else dsn.INPUT_ORDER)
        y = torch.zeros(n, N, dtype=torch.bfloat16, device=DEV)
        dsn.dsn_sliced_linear_i8(ctx, d, r, x, sx, y)
        check_status(ctx, dsn)
        return y

    near = call(x[-LAST:].clone(), sx[-LAST:].clone(), 1)
    few = call(x[-LAST:][:20].clone(), sx[-LAST:][:20].clone(), 1)
    for samples in (1, rows // 1000 if rows % 1000 == 0 else 8):
        n = rows // samples * samples
        y = call(x[rows - n:], sx[rows - n:], samples)
        assert torch.equal(y[-LAST:], near) and torch.equal(y[-LAST:][:20], few)
        del y


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("D,pairs", [(64, [16, 16]), (66, [5, 7])])
def test_rotary_far_rows(dsn, in_place, D, pairs):
    need(16)
    ctx = dsn.Context(0)
    H = 20
    row = H * 3 * D
    rows = (1 << 31) // row + 1000
    x = pattern(rows, row, torch.bfloat16)
    pos = torch.arange(2 * rows, dtype=torch.int32, device=DEV).view(2, rows) % 9973
    d = lambda n: dsn.make_rotary_desc(dsn.BF16, n, H, D, [H], pairs, shared_positions=True)
    r, _ = groups(dsn, [0], 1)
    near = x[-LAST:].clone()
    dsn.dsn_rotary_axes(ctx, d(LAST), r, pos[:, -LAST:].contiguous(), near, near)
    y = x if in_place else torch.zeros_like(x)
    dsn.dsn_rotary_axes(ctx, d(rows), r, pos, x, y)
    check_status(ctx, dsn)
    # a product and a sum, fused or one after the other in the two forms: at most one step of bf16 apart
    assert bool(((y[-LAST:].float() - near.float()).abs() <= 2.0 ** -7 * near.float().abs() + 2.0 ** -20).all())
