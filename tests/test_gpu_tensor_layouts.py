"""Rows that are column ranges of wider buffers, as views: the same results as dense tensors, bit for bit; expanded and transposed ones are refused
before anything runs."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, check_status
from transformer_util import groups

pytestmark = pytest.mark.gpu
B, R, C, N = 5, 9, 64, 96


def inside(t, before=32, after=64, fill=55):
    """A view with t's values that lies inside a wider buffer, and that buffer."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + before + after), fill, dtype=t.dtype, device=DEV)
    view = wide[..., before:before + t.shape[-1]]
    view.copy_(t)
    return view, wide


def untouched(wide, width, before=32, fill=55):
    return bool((wide[..., :before] == fill).all()) and bool((wide[..., before + width:] == fill).all())


def test_column_ranges_of_wider_buffers(dsn):
    ctx = dsn.Context(0)
    g = torch.Generator().manual_seed(4)
    r, _ = groups(dsn, [0, 1, 0, 1, 1], 2)
    x, res = (torch.randn(B, R, C, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    W = torch.randint(-127, 128, (N, C), generator=g, dtype=torch.int8).to(DEV)
    sw, pos = torch.rand(N, generator=g).to(DEV) * 1e-3, torch.arange(R, dtype=torch.int32, device=DEV)

    def front(x, res, sm, q, y, W):
        pitch = lambda t: t.stride(-2)
        sc = torch.zeros(B, R, device=DEV)
        d = dsn.make_norm_desc(dsn.BF16, R, C, [40, C], ldx=pitch(x), ld_res=pitch(res), ld_sum=pitch(sm), ldq=pitch(q))
        dsn.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=sc, residual=res, sum_out=sm)
        d = dsn.make_linear_i8_desc(R, C, N, [40, C], [48, N], W, sw, ldx=pitch(q), ldw=pitch(W), ldy=pitch(y))
        dsn.dsn_sliced_linear_i8(ctx, d, r, q, sc, y)
        d = dsn.make_rotary_desc(dsn.BF16, R, 2, 16, [1, 2], [8], shared_positions=True, ldx=pitch(y), ldy=pitch(y))
        dsn.dsn_rotary_axes(ctx, d, r, pos, y, y)
        check_status(ctx, dsn)
        return sm, q, sc, y

    blank = lambda *s, dtype=torch.bfloat16: torch.full(s, 55, dtype=dtype, device=DEV)
    want = front(x, res, blank(B, R, C), blank(B, R, C, dtype=torch.int8), blank(B, R, N), W)
    views = [inside(t) for t in (x, res, blank(B, R, C), blank(B, R, C, dtype=torch.int8), blank(B, R, N), W)]
    got = front(*(v for v, _ in views))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(untouched(wide, v.shape[-1]) for v, wide in views)


def test_expanded_and_transposed_tensors_are_refused(dsn):
    ctx = dsn.Context(0)
    r, _ = groups(dsn, [0] * B, 1)
    x, q, sc = torch.ones(B, R, C, dtype=torch.bfloat16, device=DEV), torch.full((B, R, C), 9, dtype=torch.int8, device=DEV), torch.ones(B, R, device=DEV)
    y = torch.full((B, R, N), 7, dtype=torch.bfloat16, device=DEV)
    one, one_y = torch.ones(1, R, C, dtype=torch.bfloat16, device=DEV), torch.full((1, R, N), 7, dtype=torch.bfloat16, device=DEV)
    nd = dsn.make_norm_desc(dsn.BF16, R, C, [C])
    lin = lambda res=None: dsn.make_linear_i8_desc(R, C, N, [C], [N], torch.ones(N, C, dtype=torch.int8, device=DEV), torch.ones(N, device=DEV), residual=res)
    turned = torch.ones(B, C, R, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    rd = dsn.make_rotary_desc(dsn.BF16, R, 2, 32, [2], [16], vectors=1, rotated=1)
    pos = torch.zeros(R, dtype=torch.int32, device=DEV)
    before = dict(ctx.stats())
    for call in (lambda: dsn.dsn_rmsnorm_quant(ctx, nd, r, x, q=q, scale=sc, residual=one.expand(B, R, C)),
                 lambda: dsn.dsn_rmsnorm_quant(ctx, nd, r, x, q=q, scale=sc, sum_out=one.expand(B, R, C)),
                 lambda: dsn.dsn_rmsnorm_quant(ctx, nd, r, turned, q=q, scale=sc),
                 lambda: dsn.dsn_sliced_linear_i8(ctx, lin(one_y.expand(B, R, N)), r, q, sc, y),
                 lambda: dsn.dsn_sliced_linear_i8(ctx, lin(), r, q, sc, one_y.expand(B, R, N)),
                 lambda: dsn.dsn_sliced_linear_i8(ctx, lin(), r, q[:1].expand(B, R, C), sc, y),
                 lambda: dsn.dsn_rotary_axes(ctx, rd, r, pos, x, one.expand(B, R, C)),
                 lambda: dsn.dsn_rotary_axes(ctx, rd, r, pos, turned, x)):
        with pytest.raises(dsn.DsnError) as e:
            call()
        assert e.value.code == dsn.ERR_INVALID_ARG
    assert dict(ctx.stats()) == before
    assert bool((q == 9).all()) and bool((y == 7).all()) and bool((one == 1).all()) and bool((x == 1).all())
