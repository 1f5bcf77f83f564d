"""Heads with more queries than one call of the rotary positions takes (eight vectors a head): turned where they lie by a few calls a head, then plan, write and attention over the
4-bit cache, a prompt and then token by token."""
import numpy as np
import pytest
import torch

from cache_bounds import RELATIVE, relative
from cache_util import up, workspace
from gpu_util import DEV, check_status, route_on_gpu
from oracle import dsn_oracle as O
from transformer_util import values

pytestmark = pytest.mark.gpu


def turn(dsn, ctx, r, x, B, R, H, D, group, positions):
    """The queries and keys of all heads, up to eight vectors a call; v stays."""
    vec, row = group + 2, H * (group + 2) * D
    for h in range(H):
        for a in range(0, group + 1, 8):
            n = min(8, vec - a)
            d = dsn.make_rotary_desc(dsn.BF16, R, 1, D, [1], [D // 2], vectors=n, rotated=min(n, group + 1 - a), shared_positions=False, ldx=row, ldy=row)
            at = (h * vec + a) * D
            part = x[..., at:at + n * D]
            dsn.dsn_rotary_axes(ctx, d, r, positions, part, part)


@pytest.mark.parametrize("D,group,R", [(128, 8, 30), (64, 16, 9), (128, 8, 3)])
def test_prompt_then_tokens(dsn, D, group, R):
    g = np.random.default_rng(D + group)
    ctx, B, H, page, cols, n_pages = dsn.Context(0), 4, 2, 16, 6, 20
    r = route_on_gpu(dsn, ctx, np.zeros(B, np.int32), 1)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    fixed = dict(table=i32(B, cols), lengths=i32(B), placed=i32(B), pool=i32(n_pages), pool_state=i32(2))
    pages = None
    k_all, v_all = [[] for _ in range(B)], [[] for _ in range(B)]
    for call in range(4):
        rows = R if call == 0 else 1
        d = dsn.make_cache_desc(rows, H, D, [H], group=group, page=page, n_pages=n_pages, max_pages=cols)
        if pages is None:
            pages = torch.full((dsn.dsn_cache_bytes(d),), 0xff, dtype=torch.uint8, device=DEV)
        c = dsn.make_cache(pages=pages, slots=i32(B, rows), **fixed)
        if call == 0:
            dsn.dsn_cache_reset(ctx, d, c, B)
        n = g.integers(1, rows + 1, size=B)
        x0 = O.round_bf16(g.normal(size=(B, rows, H, group + 2, D)))
        x = torch.from_numpy(x0.reshape(B, rows, -1)).to(DEV).to(torch.bfloat16)
        held = fixed["lengths"].cpu().numpy().copy()
        position = held[:, None] + np.arange(rows)
        turn(dsn, ctx, r, x, B, rows, H, D, group, up(position.reshape(1, -1)))
        out = torch.full((B, rows, H * group * D), 776.0, dtype=torch.bfloat16, device=DEV)
        dsn.dsn_cache_plan(ctx, d, c, B, up(n))
        dsn.dsn_cache_write_q4(ctx, d, c, r, x)
        dsn.dsn_cache_attention_q4(ctx, d, c, r, x, out, workspace(dsn, d, B))
        check_status(ctx, dsn)
        got_x = values(x).reshape(x0.shape)
        turned = O.rotary_axes(x0, [np.broadcast_to(position[:, :, None, None], x0.shape[:4])], [D // 2])
        # each element is a sum of two products of an element and a sine or cosine, rounded once to bf16; the angle is off by 2^-20 at most
        size = np.abs(x0).max(-1, keepdims=True)
        assert np.all(np.abs(got_x - turned)[..., :group + 1, :] <= 2.0 ** -8 * np.abs(turned)[..., :group + 1, :] + 2.0 ** -16 * size[..., :group + 1, :])
        assert np.array_equal(got_x[..., group + 1, :], x0[..., group + 1, :])
        y = values(out).reshape(B, rows, H, group, D)
        outs, refs = [], []
        for i in range(B):
            stored = O.cache_values(*O.cache_round(got_x[i, :n[i], :, -2:]))
            k_all[i].append(stored[:, :, 0])
            v_all[i].append(stored[:, :, 1])
            k, v = np.concatenate(k_all[i]), np.concatenate(v_all[i])
            for h in range(H):
                for e in range(group):
                    ref, _ = O.cache_attention(got_x[i, :n[i], h, e], k[:, h], v[:, h], D ** -0.5, len(k) - n[i])
                    outs.append(y[i, :n[i], h, e].ravel())
                    refs.append(ref.ravel())
            assert np.all(y[i, n[i]:] == 776.0)
        assert relative(np.concatenate(outs), np.concatenate(refs)) <= RELATIVE
