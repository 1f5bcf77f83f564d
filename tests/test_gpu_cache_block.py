"""The 4-bit cache as a block uses it, token by token behind a prompt: norm -> QKV on codes -> rotary positions in place -> plan, write, attention -> norm -> proj
on codes.  And what the entry points refuse."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from cache_util import Pages, attention_bound, make_desc, up, workspace
from gpu_util import DEV, check_status, route_on_gpu
from transformer_util import half_step, values

pytestmark = pytest.mark.gpu


class Block:
    """Weights, cache and buffers of a block of T paths; a call appends up to R tokens to every request."""

    def __init__(self, dsn, g, B, R, H, D, group, page, heads, embed, n_pages, max_pages):
        self.dsn, self.ctx = dsn, dsn.Context(0)
        self.B, self.H, self.D, self.group, self.heads, self.embed, self.page = B, H, D, group, heads, embed, page
        self.C, vec = max(embed), group + 2
        T, N, M = len(heads), H * vec * D, H * group * D
        rnd = lambda *s: torch.from_numpy(g.normal(size=s))
        codes = lambda *s: torch.from_numpy(g.integers(-127, 128, size=s).astype(np.int8)).to(DEV)
        self.Wqkv, self.Wout = codes(N, self.C), codes(self.C, M)
        self.sw1 = (rnd(N).abs().float() * 0.02 / np.sqrt(self.C) + 1e-4).to(DEV)
        self.sw2 = (rnd(self.C).abs().float() * 0.02 / np.sqrt(M) + 1e-4).to(DEV)
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
        self.idx = np.arange(B) % T
        self.r = route_on_gpu(dsn, self.ctx, self.idx.astype(np.int32), T)
        self.table, self.lengths, self.placed, self.pool, self.state = i32(B, max_pages), i32(B), i32(B), i32(n_pages), i32(2)
        self.N, self.M, self.T, self.vec = N, M, T, vec
        self.R = None
        self.set_rows(R, n_pages, max_pages)
        self.cache = dsn.make_cache(pages=self.pages, table=self.table, lengths=self.lengths, placed=self.placed, slots=self.slots, pool=self.pool,
                                    pool_state=self.state)
        dsn.dsn_cache_reset(self.ctx, self.d, self.cache, B)

    def set_rows(self, R, n_pages=None, max_pages=None):
        """Descriptors and buffers for calls of R rows a request; the cache stays."""
        dsn, B, C = self.dsn, self.B, self.C
        if n_pages:
            self.n_pages, self.max_pages = n_pages, max_pages
        self.R = R
        self.d = dsn.make_cache_desc(R, self.H, self.D, self.heads, group=self.group, page=self.page, n_pages=self.n_pages, max_pages=self.max_pages)
        if n_pages:
            self.pages = torch.full((dsn.dsn_cache_bytes(self.d),), 0xff, dtype=torch.uint8, device=DEV)
        z = lambda w, dt: torch.zeros(B, R, w, dtype=dt, device=DEV)
        self.x, self.q, self.s = z(C, torch.bfloat16), z(C, torch.int8), torch.zeros(B, R, device=DEV)
        self.qkv, self.val, self.out = z(self.N, torch.bfloat16), z(self.H * 2 * self.D, torch.bfloat16), z(self.M, torch.bfloat16)
        self.q2, self.s2, self.y = z(self.M, torch.int8), torch.zeros(B, R, device=DEV), z(C, torch.bfloat16)
        self.slots, self.pos = torch.zeros(B, R, dtype=torch.int32, device=DEV), torch.zeros(1, B * R, dtype=torch.int32, device=DEV)
        self.ws = workspace(dsn, self.d, B)
        self.nd = dsn.make_norm_desc(dsn.BF16, R, C, self.embed)
        self.ld = dsn.make_linear_i8_desc(R, C, self.N, self.embed, [h * self.vec * self.D for h in self.heads], self.Wqkv, self.sw1)
        self.rd = dsn.make_rotary_desc(dsn.BF16, R, self.H, self.D, self.heads, [self.D // 2], vectors=self.vec, rotated=self.vec - 1, shared_positions=False)
        self.nd2 = dsn.make_norm_desc(dsn.BF16, R, self.M, [h * self.group * self.D for h in self.heads])
        self.ld2 = dsn.make_linear_i8_desc(R, self.M, C, [h * self.group * self.D for h in self.heads], self.embed, self.Wout, self.sw2)
        if not n_pages:
            self.cache = dsn.make_cache(pages=self.pages, table=self.table, lengths=self.lengths, placed=self.placed, slots=self.slots, pool=self.pool,
                                        pool_state=self.state)

    def step(self, new):
        """x is set; new [B] on the device."""
        dsn, ctx, r = self.dsn, self.ctx, self.r
        torch.add(self.lengths.view(-1, 1), torch.arange(self.R, device=DEV, dtype=torch.int32), out=self.pos.view(self.B, self.R))
        dsn.dsn_rmsnorm_quant(ctx, self.nd, r, self.x, q=self.q, scale=self.s)
        dsn.dsn_sliced_linear_i8(ctx, self.ld, r, self.q, self.s, self.qkv)
        dsn.dsn_rotary_axes(ctx, self.rd, r, self.pos, self.qkv, self.qkv)
        dsn.dsn_cache_plan(ctx, self.d, self.cache, self.B, new)
        dsn.dsn_cache_write_q4(ctx, self.d, self.cache, r, self.qkv, values=self.val)
        dsn.dsn_cache_attention_q4(ctx, self.d, self.cache, r, self.qkv, self.out, self.ws)
        dsn.dsn_rmsnorm_quant(ctx, self.nd2, r, self.out, q=self.q2, scale=self.s2)
        dsn.dsn_sliced_linear_i8(ctx, self.ld2, r, self.q2, self.s2, self.y)


@pytest.mark.parametrize("D,group,page,R", [(64, 1, 16, 7), (128, 2, 48, 60), (64, 4, 32, 200)])
def test_prompt_then_tokens(dsn, D, group, page, R):
    g = np.random.default_rng(D + R)
    B, H, heads, embed = 5, 3, [2, 3], [96, 160]
    b = Block(dsn, g, B, R, H, D, group, page, heads, embed, n_pages=60 + B * R // page, max_pages=20 + R // page)
    k_all, v_all = [[] for _ in range(B)], [[] for _ in range(B)]
    for call in range(6):
        if call == 1:
            b.set_rows(1)
        n = g.integers(1, R + 1, size=B) if call == 0 else np.ones(B, int)
        if call == 3:
            n[2] = 0                                           # a request pauses
        if call == 4:
            n[0] = -1                                          # one ends; its row is filled again in the next call
            k_all[0], v_all[0] = [], []
        b.x.copy_(torch.from_numpy(g.normal(size=(B, b.R, b.C))))
        b.out.fill_(776.0)
        b.step(up(n))
        check_status(b.ctx, dsn)
        rows = values(b.qkv).reshape(B, b.R, H, group + 2, D)
        out, val, y = values(b.out).reshape(B, b.R, H, group, D), values(b.val).reshape(B, b.R, H, 2, D), values(b.y)
        for i in range(B):
            h, m = heads[b.idx[i]], max(int(n[i]), 0)
            code, s, z = O.cache_round(rows[i, :m, :h, -2:])
            stored = O.cache_values(code, s, z)                # [m][h][2][D]
            assert np.array_equal(val[i, :m, :h], O.round_bf16(stored))
            size = O.cache_values(np.abs(code.astype(float) - 8) + 8, s, np.abs(z))
            k_all[i].append(stored[:, :, 0])
            v_all[i].append((stored[:, :, 1], size[:, :, 1]))
            k = np.concatenate(k_all[i])
            v, vs = (np.concatenate([a[j] for a in v_all[i]]) for j in range(2))
            assert int(b.lengths[i]) == len(k)
            for hd in range(h):
                for e in range(group):
                    q = rows[i, :m, hd, e]
                    ref, p = O.cache_attention(q, k[:, hd], v[:, hd], D ** -0.5, len(k) - m)
                    assert np.all(np.abs(out[i, :m, hd, e] - ref) <= attention_bound(q, k[:, hd], vs[:, hd], p, ref, D ** -0.5))
            assert np.all(out[i, m:] == 776.0) and np.all(out[i, :, h:] == 776.0)
            if m:   # proj on the codes of what came out
                c = b.q2[i, :m, :h * group * D].double().cpu().numpy()
                ref = O.linear_i8(c[None], b.s2[i:i + 1, :m].double().cpu().numpy(), b.Wout.cpu().numpy()[:, :h * group * D], b.sw2.cpu().numpy(), [0],
                                  [h * group * D], [embed[b.idx[i]]])[0, :, :embed[b.idx[i]]]
                assert np.all(np.abs(y[i, :m, :embed[b.idx[i]]] - ref) <= (half_step(torch.bfloat16) + 2.0 ** -20) * np.abs(ref) + 1e-30)
    st = b.ctx.stats()
    assert st["launches_cache_write"] == 6 and st["launches_cache_plan"] == 7 and st["launches_cache_attention"] >= 6


def test_captured_steps_go_on_where_they_stand(dsn):
    """A captured step appends a token on every replay; the same steps made one by one give the same bits."""
    runs = []
    for captured in (False, True):
        g = np.random.default_rng(5)
        b = Block(dsn, g, 9, 30, 2, 64, 2, 16, [1, 2], [64, 128], n_pages=200, max_pages=12)
        b.x.copy_(torch.from_numpy(g.normal(size=(9, 30, b.C))))
        b.step(up(g.integers(1, 31, size=9)))
        b.set_rows(1)
        one, x = up(np.ones(9)), torch.from_numpy(g.normal(size=(9, 1, b.C))).to(torch.bfloat16).to(DEV)
        b.x.copy_(x)
        torch.cuda.synchronize()
        outs = []
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                b.step(one)
            for _ in range(40):
                graph.replay()
                outs.append(b.y.clone())
        else:
            for _ in range(40):
                b.step(one)
                outs.append(b.y.clone())
        check_status(b.ctx, dsn)
        runs.append(outs + [b.lengths.clone(), b.state.clone()])
    assert all(torch.equal(a, c) for a, c in zip(*runs))


def test_two_streams_with_a_workspace_each(dsn):
    g = np.random.default_rng(6)
    ctx, sets = dsn.Context(0), []
    for R, lengths in ((1, [3000, 40, 700] * 5), (150, [900, 150, 2000])):
        pages = Pages(g, lengths, 2, 64, 16)
        d = make_desc(dsn, pages, R, [2], 2)
        r = route_on_gpu(dsn, ctx, np.zeros(len(lengths), np.int32), 1)
        c = dsn.make_cache(pages=torch.from_numpy(pages.bytes()).to(DEV), table=up(pages.table), lengths=up(pages.lengths))
        x = torch.randn(len(lengths), R, 2 * 4 * 64, device=DEV).to(torch.bfloat16)
        for _ in range(2):
            sets.append((d, r, c, x, torch.zeros(len(lengths), R, 2 * 2 * 64, dtype=torch.bfloat16, device=DEV), workspace(dsn, d, len(lengths))))
    go = lambda s, stream=None: dsn.dsn_cache_attention_q4(ctx, s[0], s[2], s[1], s[3], s[4], s[5], stream=stream)
    alone = []
    for s in sets:
        go(s)
        torch.cuda.synchronize()
        alone.append(s[4].clone())
        s[4].zero_()
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st in zip(sets, streams):
            go(s, st)
    torch.cuda.synchronize()
    check_status(ctx, dsn)
    assert all(torch.equal(a, s[4]) for a, s in zip(alone, sets))


def test_requests_that_share_pages_read_the_same(dsn):
    g = np.random.default_rng(7)
    pages = Pages(g, [320, 320], 2, 128, 32)
    pages.table[1] = pages.table[0]
    ctx = dsn.Context(0)
    d = make_desc(dsn, pages, 1, [2], 1)
    r = route_on_gpu(dsn, ctx, np.zeros(2, np.int32), 1)
    x = torch.randn(1, 1, 2 * 3 * 128, device=DEV).to(torch.bfloat16).expand(2, 1, -1).contiguous()
    out = torch.zeros(2, 1, 256, dtype=torch.bfloat16, device=DEV)
    dsn.dsn_cache_attention_q4(ctx, d, dsn.make_cache(pages=torch.from_numpy(pages.bytes()).to(DEV), table=up(pages.table), lengths=up(pages.lengths)), r, x, out,
                               workspace(dsn, d, 2))
    check_status(ctx, dsn)
    assert torch.equal(out[0], out[1]) and bool(out.any())


def test_pages_beyond_two_to_the_31_bytes(dsn):
    """Pages at the end of a pool of 2.65e9 bytes, for the few-queries and the many-rows form."""
    g = np.random.default_rng(8)
    small = Pages(g, [600, 300], 8, 128, 256)
    n_pages = 9000
    per = 8 * 16 * 18 * 128
    pool = torch.zeros(n_pages * per, dtype=torch.uint8, device=DEV)
    raw = torch.from_numpy(small.bytes()).to(DEV).view(small.n_pages, per)
    shift = n_pages - small.n_pages
    pool.view(n_pages, per)[shift:] = raw
    table = np.where(small.table >= 0, small.table + shift, -1)
    ctx = dsn.Context(0)
    r = route_on_gpu(dsn, ctx, np.zeros(2, np.int32), 1)
    for R in (1, 40):
        x = torch.randn(2, R, 8 * 3 * 128, device=DEV).to(torch.bfloat16)
        got = []
        for pg, tb, n in ((pool, table, n_pages), (raw.flatten(), small.table, small.n_pages)):
            d = dsn.make_cache_desc(R, 8, 128, [8], page=256, n_pages=n, max_pages=small.max_pages)
            out = torch.zeros(2, R, 8 * 128, dtype=torch.bfloat16, device=DEV)
            dsn.dsn_cache_attention_q4(ctx, d, dsn.make_cache(pages=pg, table=up(tb), lengths=up(small.lengths)), r, x, out, workspace(dsn, d, 2))
            got.append(out)
        check_status(ctx, dsn)
        assert torch.equal(*got) and bool(got[0].any())


# ---------------------------------------------------------------------------------------------- refusals of the library itself
def test_refusals(dsn):
    ctx = dsn.Context(0)
    B, R, H, D, G, n_pages, cols = 2, 3, 2, 64, 2, 6, 4
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    desc = lambda **kw: dsn.make_cache_desc(**{**dict(R=R, H=H, D_h=D, heads=[H], group=G, page=16, n_pages=n_pages, max_pages=cols), **kw})
    t = dict(pages=torch.zeros(n_pages * H * 1152 + 16, dtype=torch.uint8, device=DEV), table=i32(B, cols), lengths=i32(B), placed=i32(B), slots=i32(B, R),
             pool=i32(n_pages), pool_state=i32(2))
    full = dsn.make_cache(**t)
    r = route_on_gpu(dsn, ctx, np.zeros(B, np.int32), 1)
    x, out, val = (torch.zeros(B, R, w, dtype=torch.bfloat16, device=DEV) for w in (H * (G + 2) * D, H * G * D, H * 2 * D))
    ws = workspace(dsn, desc(), B)
    new = i32(B)
    lib = ctx.lib
    P = lambda a: None if a is None else a.data_ptr()
    reset = lambda d=None, c=full, n=B: lib.dsn_cache_reset(ctx.handle, d or desc(), c, n, None)
    plan = lambda d=None, c=full, n=B, nt=new, lo=None: lib.dsn_cache_plan(ctx.handle, d or desc(), c, n, P(nt), P(lo), None, None)
    write = lambda d=None, c=full, r=r, a=x, v=val: lib.dsn_cache_write_q4(ctx.handle, d or desc(), c, r, P(a), P(v), None)
    attend = lambda d=None, c=full, r=r, a=x, o=out, w=ws, n=None: lib.dsn_cache_attention_q4(ctx.handle, d or desc(), c, r, P(a), P(o), P(w),
                                                                                             (0 if w is None else w.numel()) if n is None else n, None)
    assert reset() == plan() == write() == attend() == 0
    before = ctx.stats()["launches"]
    for bad in (dict(R=0), dict(D_h=96), dict(group=65), dict(page=24), dict(n_pages=2 ** 30), dict(heads=[3]), dict(heads=[0]), dict(order=7), dict(window=-1),
                dict(scale=float("nan"))):
        for call in (reset, plan, write, attend):
            assert call(d=desc(**bad)) == dsn.ERR_INVALID_ARG, bad
    assert attend(d=desc(R=2 ** 24, max_pages=2 ** 20)) == dsn.ERR_UNSUPPORTED
    f32 = desc()
    f32.dtype = dsn.F32
    assert write(d=f32) == attend(d=f32) == dsn.ERR_INVALID_ARG
    for name, calls in (("pages", (write, attend)), ("table", (plan, attend)), ("lengths", (reset, plan, attend)), ("placed", (plan,)), ("slots", (plan, write)),
                        ("pool", (reset, plan)), ("pool_state", (reset, plan))):
        part = dsn.make_cache(**{k: v for k, v in t.items() if k != name})
        for call in calls:
            assert call(c=part) == dsn.ERR_INVALID_ARG, name
    none = ctypes.POINTER(dsn.Cache)()
    for call in (reset, plan, write, attend):
        assert call(c=none) == dsn.ERR_INVALID_ARG
    assert plan(nt=None) == plan(n=-1) == reset(n=-1) == dsn.ERR_INVALID_ARG
    assert plan(nt=t["placed"]) == plan(nt=t["slots"]) == plan(lo=new) == plan(lo=t["placed"]) == dsn.ERR_INVALID_ARG
    assert write(a=None) == attend(a=None) == attend(o=None) == dsn.ERR_INVALID_ARG
    assert write(v=x) == attend(o=x) == dsn.ERR_INVALID_ARG
    for kw in (dict(ld_qkv=H * (G + 2) * D - 8),):
        assert write(d=desc(**kw)) == attend(d=desc(**kw)) == dsn.ERR_INVALID_ARG
    assert write(d=desc(ld_values=8)) == attend(d=desc(ld_out=8)) == dsn.ERR_INVALID_ARG
    for kw in (dict(ld_qkv=H * (G + 2) * D + 4),):
        assert write(d=desc(**kw)) == attend(d=desc(**kw)) == dsn.ERR_ALIGNMENT
    odd = lambda a: a.flatten()[1:]
    assert write(a=odd(x)) == write(v=odd(val)) == attend(a=odd(x)) == attend(o=odd(out)) == dsn.ERR_ALIGNMENT
    assert write(c=dsn.make_cache(**{**t, "pages": t["pages"][8:]})) == attend(c=dsn.make_cache(**{**t, "pages": t["pages"][8:]})) == dsn.ERR_ALIGNMENT
    assert attend(w=None) == attend(n=ws.numel() - 1) == dsn.ERR_WORKSPACE
    assert attend(w=ws[8:]) == dsn.ERR_ALIGNMENT
    bad_r = dsn.make_routing(B, 2, i32(2), i32(3), i32(2), i32(2))
    assert write(r=bad_r) == attend(r=bad_r) == dsn.ERR_INVALID_ARG                     # more groups than paths
    assert ctx.stats()["launches"] == before and ctx.get_status()[0] == 0
    empty = dsn.make_routing(0, 1, i32(1), i32(2), i32(1), i32(1))
    assert write(r=empty) == attend(r=empty, w=None) == reset(n=0) == 0
