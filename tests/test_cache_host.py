"""4-bit cache on the host: the oracle's forms against independent ones, descriptor layouts, sizes, and what the binding refuses.  No GPU."""
import ctypes
import os
import subprocess
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2109_10060_b200.build import build
    build()
    import paper_2109_10060_b200 as dsn
    return dsn


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


class OnNextGpu(torch.Tensor):
    def get_device(self):
        return 1


def on(t, cls=OnGpu):
    return t.as_subclass(cls)


# ---------------------------------------------------------------------------------------------- the oracle
def test_rounding_is_to_the_nearest_step_of_its_own_grid():
    g = np.random.default_rng(1)
    x = O.round_bf16(g.normal(size=(5, 3, 128)) * np.exp(g.normal(size=(5, 3, 1))))
    code, s, z = O.cache_round(x)
    assert code.shape == (5, 3, 2, 64) and s.shape == z.shape == (5, 3, 2) and code.max() == 15 and code.min() == 0
    v = O.cache_values(code, s, z)
    grid = z[..., None, None] + s[..., None, None] * (np.arange(16) - 8)                        # [..., 1, 16]
    best = np.abs(x.reshape(5, 3, 2, 64, 1) - grid).min(-1)
    # a tie between two steps may go either way, and the product with 1 / scale is off by 2^-23 of a code
    assert np.all(np.abs(x - v).reshape(best.shape) <= best + s[..., None] * 16 * 2.0 ** -22)


def test_rounding_of_constant_and_tiny_groups():
    for c in (0.0, 3.0, -2.0 ** -130):
        code, s, z = O.cache_round(np.full(64, c))
        assert np.all(code == 8) and s[0] == 0 and z[0] == c
    assert np.all(O.cache_values(*O.cache_round(np.linspace(-1, 1, 64).astype(np.float32))) < 1.1)


def test_places_of_elements_do_not_meet():
    D, page, H = 128, 48, 3
    seen = set()
    for slot in range(2 * page):
        for head in range(H):
            for half in range(2):
                for group in range(2):
                    for e in range(64):
                        byte, shift, pair = O.cache_place(D, page, H, slot, head, half, group, e)
                        assert (byte, shift) not in seen
                        seen.add((byte, shift))
                    for b in range(4):
                        assert (pair + b, "pair") not in seen and (pair + b, 0) not in seen
                        seen.add((pair + b, "pair"))
    used = {b for b, _ in seen}
    assert used == set(range(2 * H * (page // 16) * 18 * D))                                     # no byte left over


def test_attention_against_library_and_by_differences():
    g = np.random.default_rng(2)
    q, k, v = g.normal(size=(5, 8)), g.normal(size=(9, 8)), g.normal(size=(9, 3))
    out, p = O.cache_attention(q, k, v, 0.3, 4)
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(a)[None] for a in (q, k, v)), scale=0.3,
                                                           attn_mask=torch.from_numpy(np.arange(9)[None, :] <= 4 + np.arange(5)[:, None])[None])
    np.testing.assert_allclose(out, ref[0].numpy(), rtol=1e-12)
    np.testing.assert_allclose(p.sum(-1), 1)
    win, pw = O.cache_attention(q, k, v, 0.3, 4, window=2)
    assert np.all((pw > 0).sum(-1) == 2)
    np.testing.assert_allclose(win[0], O.cache_attention(q[:1], k[3:5], v[3:5], 0.3, 1)[0][0])
    assert np.all(O.cache_attention(q, k, v, 0.3, -5)[0] == 0)                                   # nothing seen
    h = 1e-6                                                                                     # d out / d v is p
    d = (O.cache_attention(q, k, v + h, 0.3, 4)[0] - out) / h
    np.testing.assert_allclose(d, 1, rtol=1e-6)


def test_plan_of_the_oracle_keeps_every_page_once():
    g = np.random.default_rng(3)
    B, R, page, N = 7, 40, 16, 30
    held, table, ring, first, free = [0] * B, [[] for _ in range(B)], list(range(N)), 0, N
    for _ in range(40):
        new = [int(n) for n in g.integers(-1, R + 1, size=B)]
        placed, held, table, slots, ring, first, free, full, bad = O.cache_plan(held, new, table, ring, first, free, page, 6, R)
        assert not bad
        table = [t[:-(-h // page)] for t, h in zip(table, held)]
        owned = [p for t in table for p in t]
        assert sorted(owned + [ring[(first + j) % N] for j in range(free)]) == list(range(N))
        for i in range(B):
            assert sum(s >= 0 for s in slots[i]) == placed[i]


# ---------------------------------------------------------------------------------------------- the binding
def test_descriptor_layouts(lib, tmp_path):
    names = {"dsn_cache_desc": lib.CacheDesc, "dsn_cache": lib.Cache, "dsn_stats": lib.Stats}
    body = "".join(f'printf("{n} %zu\\n", sizeof({n}));' for n in names)
    for n, cls in names.items():
        body += "".join(f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));' for f, _ in cls._fields_)
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dsn.h"\nint main(void){' + body + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    out = subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()
    got = dict(zip(out[0::2], map(int, out[1::2])))
    for n, cls in names.items():
        assert got[n] == ctypes.sizeof(cls), n
        for f, _ in cls._fields_:
            assert got[f"{n}.{f}"] == getattr(cls, f).offset, f"{n}.{f}"


def test_sizes(lib):
    d = lib.make_cache_desc(1, 8, 128, [8], group=4, page=48, n_pages=100, max_pages=10)
    assert lib.dsn_cache_bytes(d) == 100 * 8 * 3 * 18 * 128
    few = lib.dsn_cache_attention_q4_workspace_bytes(d, 3)
    assert few > 0 and lib.dsn_cache_attention_q4_workspace_bytes(d, 1000) > few
    many = lib.make_cache_desc(500, 8, 128, [8], group=4, page=48, n_pages=100, max_pages=10)
    assert lib.dsn_cache_attention_q4_workspace_bytes(many, 3) > 0
    big = lib.make_cache_desc(1, 4096, 128, [4096], page=1024, n_pages=2 ** 20, max_pages=2 ** 19)
    assert lib.dsn_cache_bytes(big) == 2 ** 20 * 4096 * 64 * 18 * 128                            # beyond 32 bits
    assert lib.dsn_cache_attention_q4_workspace_bytes(d, -1) == 0


WRONG = [dict(R=0), dict(R=2 ** 24 + 1), dict(H=0), dict(H=4097), dict(D_h=32), dict(D_h=96), dict(D_h=256), dict(group=0), dict(group=65), dict(page=0),
         dict(page=8), dict(page=24), dict(page=1040), dict(n_pages=0), dict(n_pages=2 ** 30), dict(max_pages=0), dict(max_pages=2 ** 28), dict(heads=[]),
         dict(heads=[0]), dict(heads=[5]), dict(heads=[1] * 65), dict(order=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1),
         dict(R=2 ** 24, max_pages=2 ** 20)]


@pytest.mark.parametrize("change", WRONG)
def test_descriptors_that_are_not_valid_have_no_size(lib, change):
    good = dict(R=2, H=4, D_h=64, heads=[1, 4], group=2, page=16, n_pages=10, max_pages=4)
    assert lib.dsn_cache_bytes(lib.make_cache_desc(**good)) > 0
    bad = lib.make_cache_desc(**{**good, **change})
    assert lib.dsn_cache_bytes(bad) == 0 and lib.dsn_cache_attention_q4_workspace_bytes(bad, 1) == 0


class Calls:
    """A context whose library records the calls that get through."""

    def __init__(self, device=0):
        self.seen = []
        self.handle, self.device = ctypes.c_void_p(), device
        self.lib = SimpleNamespace(**{n: self.record for n in ("dsn_cache_reset", "dsn_cache_plan", "dsn_cache_write_q4", "dsn_cache_attention_q4")})

    def record(self, *a):
        self.seen.append(a)
        return 0


STREAM = SimpleNamespace(cuda_stream=0)
B, R, H, D, G, PAGES, COLS = 3, 4, 2, 64, 2, 9, 5


def tensors(**change):
    i32 = lambda *s: on(torch.zeros(*s, dtype=torch.int32))
    t = dict(pages=on(torch.zeros(PAGES * H * 1152, dtype=torch.uint8)), table=i32(B, COLS), lengths=i32(B), placed=i32(B), slots=i32(B, R), pool=i32(PAGES),
             pool_state=i32(2))
    t.update(change)
    return t


def setting(lib, **change):
    a = on(torch.zeros(B + 1, dtype=torch.int32))
    d = lib.make_cache_desc(R, H, D, [H], group=G, page=16, n_pages=PAGES, max_pages=COLS)
    bf = lambda w: on(torch.zeros(B, R, w, dtype=torch.bfloat16))
    return d, lib.make_cache(**tensors(**change)), lib.make_routing(B, 1, a, a, a, a), bf(H * (G + 2) * D), bf(H * G * D), bf(H * 2 * D)


def all_calls(lib, ctx, d, c, r, qkv, out, values, new=None, ws=None):
    new = on(torch.zeros(B, dtype=torch.int32)) if new is None else new
    return [lambda: lib.dsn_cache_reset(ctx, d, c, B, stream=STREAM), lambda: lib.dsn_cache_plan(ctx, d, c, B, new, stream=STREAM),
            lambda: lib.dsn_cache_write_q4(ctx, d, c, r, qkv, values=values, stream=STREAM),
            lambda: lib.dsn_cache_attention_q4(ctx, d, c, r, qkv, out, ws, stream=STREAM)]


def test_calls_with_everything_in_order_get_through(lib):
    ctx = Calls()
    for call in all_calls(lib, ctx, *setting(lib)):
        call()
    assert len(ctx.seen) == 4


@pytest.mark.parametrize("name,calls", [("pages", (2, 3)), ("table", (1, 3)), ("lengths", (0, 1, 3)), ("placed", (1, 3)), ("slots", (1, 2)), ("pool", (0, 1)),
                                        ("pool_state", (0, 1))])
def test_a_tensor_that_is_too_small_is_refused_where_it_is_used(lib, name, calls):
    ctx = Calls()
    t = tensors()[name]
    cases = all_calls(lib, ctx, *setting(lib, **{name: t.flatten()[:-1].contiguous().as_subclass(OnGpu)}))
    for i, call in enumerate(cases):
        if i in calls:
            with pytest.raises(lib.DsnError) as e:
                call()
            assert e.value.code == lib.ERR_INVALID_ARG and name in str(e.value)
        else:
            call()


def test_tensors_of_another_type_layout_or_device_are_refused(lib):
    for name in ("table", "lengths", "placed", "slots", "pool", "pool_state"):
        for wrong in (on(torch.zeros(50, dtype=torch.int64)), on(torch.zeros(50, 2, dtype=torch.int32).t()), torch.zeros(50, dtype=torch.int32)):
            with pytest.raises(lib.DsnError):
                lib.make_cache(**tensors(**{name: wrong}))
    with pytest.raises(lib.DsnError):
        lib.make_cache(**tensors(pages=on(torch.zeros(10000, dtype=torch.float32))))
    with pytest.raises(lib.DsnError):
        lib.make_cache(**tensors(pool=on(torch.zeros(PAGES, dtype=torch.int32), OnNextGpu)))     # not all on one GPU
    ctx = Calls(device=1)
    for call in all_calls(lib, ctx, *setting(lib)):
        with pytest.raises(lib.DsnError):
            call()
    ctx = Calls()
    d, c, r, qkv, out, values = setting(lib)
    short = lambda t: on(torch.zeros(B, R, t.shape[-1] - 8, dtype=torch.bfloat16))
    half = lambda t: on(t.as_subclass(torch.Tensor).to(torch.float16))
    wide = lambda t: on(torch.zeros(B, R, 2 * t.shape[-1], dtype=torch.bfloat16))[..., ::2]
    for f in (short, half, wide, lambda t: t.as_subclass(torch.Tensor)):
        with pytest.raises(lib.DsnError):
            lib.dsn_cache_write_q4(ctx, d, c, r, f(qkv), values=values, stream=STREAM)
        with pytest.raises(lib.DsnError):
            lib.dsn_cache_write_q4(ctx, d, c, r, qkv, values=f(values), stream=STREAM)
        with pytest.raises(lib.DsnError):
            lib.dsn_cache_attention_q4(ctx, d, c, r, f(qkv), out, stream=STREAM)
        with pytest.raises(lib.DsnError):
            lib.dsn_cache_attention_q4(ctx, d, c, r, qkv, f(out), stream=STREAM)
    for ws in (torch.zeros(64, dtype=torch.uint8), on(torch.zeros(64, 2, dtype=torch.uint8).t())):
        with pytest.raises(lib.DsnError):
            lib.dsn_cache_attention_q4(ctx, d, c, r, qkv, out, ws, stream=STREAM)
    for new in (on(torch.zeros(B, dtype=torch.int64)), on(torch.zeros(B - 1, dtype=torch.int32)), torch.zeros(B, dtype=torch.int32)):
        with pytest.raises(lib.DsnError):
            lib.dsn_cache_plan(ctx, d, c, B, new, stream=STREAM)
    assert not ctx.seen


def test_strided_rows_get_through(lib):
    ctx = Calls()
    d, c, r, qkv, out, values = setting(lib)
    w = H * (G + 2) * D
    d2 = lib.make_cache_desc(R, H, D, [H], group=G, page=16, n_pages=PAGES, max_pages=COLS, ld_qkv=w + 64)
    view = on(torch.zeros(B, R, w + 64, dtype=torch.bfloat16))[..., :w]
    lib.dsn_cache_write_q4(ctx, d2, c, r, view, stream=STREAM)
    lib.dsn_cache_attention_q4(ctx, d2, c, r, view, out, stream=STREAM)
    assert len(ctx.seen) == 2
