"""The 8-bit operators together, as the front of a slimmable transformer block uses them: residual + norm + codes (gathered to grouped
order) -> QKV on codes -> rotary positions of a token grid in place -> the sliced attention core."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV, check_status, route_on_gpu
from transformer_util import half_step, values

pytestmark = pytest.mark.gpu


def grid_positions(side, prefix):
    """Height and width of the tokens of a square image behind `prefix` tokens at the origin."""
    p = np.zeros((2, prefix + side * side), np.int32)
    p[0, prefix:], p[1, prefix:] = np.repeat(np.arange(side), side), np.tile(np.arange(side), side)
    return p


@pytest.mark.parametrize("B,side", [(24, 14), (2, 3), (300, 7)])
def test_block_front_matches_oracle_and_replays(dsn, B, side):
    g = np.random.default_rng(B)
    ctx = dsn.Context(0)
    N, De, H, Dh = 1 + side * side, 384, 6, 64
    embed, heads = [192, 288, 384], [3, 4, 6]
    T = len(heads)
    idx = g.integers(0, T, size=B).astype(np.int32)
    r = route_on_gpu(dsn, ctx, idx, T)
    perm = O.route(idx, T)[2]
    x, res = (torch.from_numpy(g.normal(size=(B, N, De))).to(torch.bfloat16) for _ in range(2))
    w = g.uniform(0.5, 1.5, De).astype(np.float32)
    W = g.integers(-127, 128, size=(3 * H * Dh, De)).astype(np.int8)
    sw = (g.uniform(0.5, 1.5, 3 * H * Dh) / 73 / np.sqrt(De)).astype(np.float32)
    bias = (0.1 * g.normal(size=3 * H * Dh)).astype(np.float32)
    pos = grid_positions(side, 1)
    pairs = [16, 16]
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    xd, rd, sum_, wd, Wd, swd, bd, pd = x.to(DEV), res.to(DEV), torch.zeros_like(x, device=DEV), up(w), up(W), up(sw), up(bias), up(pos)
    q, sc = torch.zeros(B, N, De, dtype=torch.int8, device=DEV), torch.zeros(B, N, device=DEV)
    qkv = torch.zeros(B, N, 3 * H * Dh, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(B, N, H * Dh, dtype=torch.bfloat16, device=DEV)
    nd = dsn.make_norm_desc(dsn.BF16, N, De, embed, wd, out_order=dsn.GROUPED)
    ld = dsn.make_linear_i8_desc(N, De, 3 * H * Dh, embed, [3 * Dh * h for h in heads], Wd, swd, bias=bd, in_order=dsn.GROUPED, out_order=dsn.GROUPED)
    pdsc = dsn.make_rotary_desc(dsn.BF16, N, H, Dh, heads, pairs, ladder=dsn.ROTARY_PER_AXIS, shared_positions=True, order=dsn.GROUPED)
    ad = dsn.make_attention_desc(N, H, Dh, heads, order=dsn.GROUPED)

    def block():
        dsn.dsn_rmsnorm_quant(ctx, nd, r, xd, q=q, scale=sc, residual=rd, sum_out=sum_)
        dsn.dsn_sliced_linear_i8(ctx, ld, r, q, sc, qkv)
        dsn.dsn_rotary_axes(ctx, pdsc, r, pd, qkv, qkv)
        dsn.dsn_sliced_attention(ctx, ad, r, qkv, out)

    block()
    check_status(ctx, dsn)
    got, codes, scales, turned = values(out), values(q), values(sc), values(qkv)
    path = idx[perm]
    xin, rin = x.double().numpy()[perm], res.double().numpy()[perm]
    _, _, scale, steps = O.rmsnorm_quant(xin, path, embed, w.astype(np.float64), 1e-6, rin)
    worst = 0.0
    for i in range(B):
        e, h = embed[path[i]], heads[path[i]]
        assert np.all(np.abs(codes[i, :, :e] - steps[i, :, :e]) <= 0.5 + 127 * 7 * 2.0 ** -24)
        # from the codes on: QKV and the turned vectors are stored in bf16, so the mirror rounds there too
        y = O.linear_i8(codes[i:i + 1, :, :e], scales[i:i + 1], W[:, :e], sw, [0], [e], [3 * Dh * h], bias)[0, :, :3 * Dh * h]
        y = O.round_bf16(y).reshape(N, h, 3, Dh)
        p = np.broadcast_to(pos[:, :, None, None], (2, N, h, 2))
        y[:, :, :2] = O.round_bf16(O.rotary_axes(y[:, :, :2], p, pairs, per_axis=True))
        # a stored value differs from the mirror's by a step where the two fell on different sides of a border, once in the product and once in
        # the turn of its two elements: at most 3 steps of the pair's larger value
        mine = turned[i, :, :3 * Dh * h].reshape(N, h, 3, Dh)
        big = np.maximum(np.abs(y), np.concatenate([np.abs(y[..., 32:]), np.abs(y[..., :32])], -1))
        assert np.all(np.abs(mine - y) <= 3 * 2 * half_step(torch.bfloat16) * big + 1e-30)
        ref = O.attention(*(mine[:, :, j].reshape(1, N, h * Dh) for j in range(3)), [0], [h], Dh)[0]
        err = np.max(np.abs(got[i, :, :h * Dh] - ref)) / np.max(np.abs(ref))
        worst = max(worst, err)
        assert err <= 5e-3                                     # the attention core's own bound
        assert np.all(got[i, :, h * Dh:] == 0)
    first = [t.clone() for t in (q, sc, qkv, out, sum_)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for t in (q, sc, qkv, out, sum_):
        t.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (q, sc, qkv, out, sum_)))
    st = ctx.stats()
    assert st["launches_norm"] == 2 and st["launches_rotary"] == 2 and st["launches_gemm_i8"] + st["launches_rows_i8"] == 2


def test_two_streams_on_one_context_do_not_disturb_each_other(dsn):
    ctx = dsn.Context(0)
    g = torch.Generator().manual_seed(3)
    r = route_on_gpu(dsn, ctx, np.zeros(64, np.int32), 1)
    N, C = 40, 512
    W = torch.randint(-127, 128, (640, C), generator=g, dtype=torch.int8).to(DEV)
    sw = torch.rand(640, generator=g).to(DEV) * 1e-3
    nd = dsn.make_norm_desc(dsn.BF16, N, C, [C])
    ld = dsn.make_linear_i8_desc(N, C, 640, [C], [640], W, sw)
    pd = dsn.make_rotary_desc(dsn.BF16, N, 10, 64, [10], [32], vectors=1, rotated=1, shared_positions=True)
    pos = torch.arange(N, dtype=torch.int32, device=DEV)

    def buffers(seed):
        x = torch.randn(64, N, C, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)
        return x, torch.zeros(64, N, C, dtype=torch.int8, device=DEV), torch.zeros(64, N, device=DEV), torch.zeros(64, N, 640, dtype=torch.bfloat16, device=DEV)

    def go(b, s):
        dsn.dsn_rmsnorm_quant(ctx, nd, r, b[0], q=b[1], scale=b[2], stream=s)
        dsn.dsn_sliced_linear_i8(ctx, ld, r, b[1], b[2], b[3], stream=s)
        dsn.dsn_rotary_axes(ctx, pd, r, pos, b[3], b[3], stream=s)

    alone = []
    for seed in (1, 2):
        b = buffers(seed)
        go(b, None)
        torch.cuda.synchronize()
        alone.append(b[3].clone())
    sets, streams = [buffers(1), buffers(2)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(sets, streams):
            go(b, s)
    torch.cuda.synchronize()
    check_status(ctx, dsn)
    assert all(torch.equal(a, b[3]) for a, b in zip(alone, sets))
