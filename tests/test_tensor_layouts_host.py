"""Which tensors the binding of the 8-bit transformer operators hands to the library: strides, storage and device.  No GPU: host tensors that say
they lie on one, and a library that only records its calls."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

STREAM = SimpleNamespace(cuda_stream=0)


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


class OnNextGpu(torch.Tensor):
    def get_device(self):
        return 1


def on(t, cls=OnGpu):
    return t.as_subclass(cls)


@pytest.fixture(scope="module")
def lib():
    from paper_2109_10060_b200.build import build
    build()
    import paper_2109_10060_b200 as dsn
    return dsn


class Calls:
    """Records the pointers of every call that gets through."""

    def __init__(self, device=0):
        self.seen = []
        self.handle, self.device = ctypes.c_void_p(), device
        self.lib = SimpleNamespace(**{n: self.record for n in ("dsn_rmsnorm_quant", "dsn_sliced_linear_i8", "dsn_rotary_axes")})

    def record(self, ctx, d, routing, *pointers):
        self.seen.append(pointers)
        return 0


def routing(lib, B):
    a = torch.zeros(B + 1, dtype=torch.int32)
    return lib.make_routing(B, 1, a, a, a, a)


B, R, C = 6, 4, 32


def layouts(dt, width=C):
    """(tensor, leading dimension, accepted) of [B][R][width] rows."""
    one = torch.zeros(1, 1, width, dtype=dt)
    wide = torch.zeros(B, R, 3 * width, dtype=dt)
    return [
        (torch.zeros(B, R, width, dtype=dt), width, True),
        (torch.zeros(B * R * width + 5, dtype=dt), width, True),                        # a flat buffer
        (wide, 3 * width, True),
        (wide[..., width:2 * width], 3 * width, True),                                  # a range of columns
        (wide.view(B, R, 3, 2, width // 2)[:, :, 1], 3 * width, True),                  # the same, its columns split
        (wide[..., 2 * width:].view(B * R, width), 3 * width, True),
        (torch.zeros(B, R, width, dtype=dt)[:, :, ::1], width, True),
        (one.expand(B, R, width), width, False),                                        # one stored row
        (torch.zeros(1, R, width, dtype=dt).expand(B, R, width), width, False),         # one stored sample
        (torch.zeros(B, 1, width, dtype=dt).expand(B, R, width), width, False),
        (torch.zeros(B, R, 1, dtype=dt).expand(B, R, width), width, False),
        (torch.zeros(B, width, R, dtype=dt).transpose(1, 2), width, False),             # columns before rows
        (torch.zeros(R, B, width, dtype=dt).transpose(0, 1), width, False),             # rows before samples
        (torch.zeros(B, 2 * R, width, dtype=dt)[:, :R], width, False),                  # a gap behind every sample
        (torch.zeros(B, R, 2 * width, dtype=dt)[..., ::2], 2 * width, False),
        (wide[..., :width], width, False),                                              # rows further apart than the descriptor says
        (wide[..., :width], 6 * width, False),
        (wide[1:, ..., width:], 3 * width, False),                                      # a sample short
        (torch.zeros(B * R * width - 1, dtype=dt), width, False),
    ]


def outcome(lib, ctx, call):
    try:
        call()
    except lib.DsnError as e:
        assert e.code == lib.ERR_INVALID_ARG
        return False
    return True


@pytest.mark.parametrize("what", ["x", "residual", "sum_out", "q", "y"])
def test_norm_takes_rows_and_nothing_else(lib, what):
    dt, i8 = torch.bfloat16, torch.int8
    for t, ld, fine in layouts(i8 if what == "q" else dt):
        full = dict(x=torch.zeros(B, R, C, dtype=dt), residual=torch.zeros(B, R, C, dtype=dt), sum_out=torch.zeros(B, R, C, dtype=dt),
                    q=torch.zeros(B, R, C, dtype=i8), y=torch.zeros(B, R, C, dtype=dt), scale=torch.zeros(B, R))
        full[what] = t
        full = {k: on(v) for k, v in full.items()}
        d = lib.make_norm_desc(lib.BF16, R, C, [C], **{dict(x="ldx", residual="ld_res", sum_out="ld_sum", q="ldq", y="ldy")[what]: ld})
        ctx = Calls()
        got = outcome(lib, ctx, lambda: lib.dsn_rmsnorm_quant(ctx, d, routing(lib, B), full.pop("x"), stream=STREAM, **full))
        assert got == fine == (len(ctx.seen) == 1), (what, tuple(t.shape), t.stride(), ld)
        if fine:
            assert t.data_ptr() in ctx.seen[0]


@pytest.mark.parametrize("what", ["x", "residual", "y", "W"])
def test_linear_takes_rows_and_nothing_else(lib, what):
    dt, i8, N = torch.bfloat16, torch.int8, 32
    for t, ld, fine in layouts(dt if what in ("residual", "y") else i8):
        full = dict(x=torch.zeros(B, R, C, dtype=i8), residual=torch.zeros(B, R, N, dtype=dt), y=torch.zeros(B, R, N, dtype=dt),
                    W=torch.zeros(B * R, C, dtype=i8))
        lds = dict(ldx=C, ldw=C, ldy=N)
        lds[dict(x="ldx", W="ldw").get(what, "ldy")] = ld
        if what in ("residual", "y"):                            # the two share their leading dimension
            full["y" if what == "residual" else "residual"] = torch.zeros(B, R, ld, dtype=dt)
        full[what] = t
        full = {k: on(v) for k, v in full.items()}
        ctx = Calls()

        def call():
            out = B * R if what == "W" else N
            lds["ldy"] = max(lds["ldy"], out) if what == "W" else lds["ldy"]
            d = lib.make_linear_i8_desc(R, C, out, [C], [out], full["W"] if what == "W" else on(torch.zeros(N, C, dtype=i8)), on(torch.ones(out)),
                                        residual=full["residual"], **lds)
            lib.dsn_sliced_linear_i8(ctx, d, routing(lib, B), full["x"], on(torch.zeros(B, R)), full["y"], stream=STREAM)

        assert outcome(lib, ctx, call) == fine == (len(ctx.seen) == 1), (what, tuple(t.shape), t.stride(), ld)


@pytest.mark.parametrize("what", ["x", "y"])
def test_rotary_takes_rows_and_nothing_else(lib, what):
    for t, ld, fine in layouts(torch.bfloat16):
        full = dict(x=torch.zeros(B, R, C, dtype=torch.bfloat16), y=torch.zeros(B, R, C, dtype=torch.bfloat16))
        full[what] = t
        d = lib.make_rotary_desc(lib.BF16, R, 2, 16, [2], [8], vectors=1, rotated=1, **{"ld" + what: ld})
        ctx = Calls()
        got = outcome(lib, ctx, lambda: lib.dsn_rotary_axes(ctx, d, routing(lib, B), on(torch.zeros(R, dtype=torch.int32)), on(full["x"]), on(full["y"]),
                                                            stream=STREAM))
        assert got == fine == (len(ctx.seen) == 1), (what, tuple(t.shape), t.stride(), ld)


def test_dense_arguments_and_workspace_may_not_be_expanded(lib):
    x, q, y = (on(torch.zeros(B, R, C, dtype=t)) for t in (torch.bfloat16, torch.int8, torch.bfloat16))
    r, ctx = routing(lib, B), Calls()
    scale = on(torch.zeros(B, 1).expand(B, R))
    w = on(torch.zeros(1).expand(C))
    d = lib.make_norm_desc(lib.BF16, R, C, [C])
    l = lib.make_linear_i8_desc(R, C, C, [C], [C], on(torch.zeros(C, C, dtype=torch.int8)), on(torch.ones(C)))
    p = lib.make_rotary_desc(lib.BF16, R, 2, 16, [2], [8], vectors=1, rotated=1)
    for call in (lambda: lib.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=scale, stream=STREAM),
                 lambda: lib.make_norm_desc(lib.BF16, R, C, [C], w),
                 lambda: lib.make_linear_i8_desc(R, C, C, [C], [C], on(torch.zeros(C, C, dtype=torch.int8)), w),
                 lambda: lib.dsn_sliced_linear_i8(ctx, l, r, q, scale, y, stream=STREAM),
                 lambda: lib.dsn_sliced_linear_i8(ctx, l, r, q, on(torch.zeros(B, R)), y, on(torch.zeros(1, dtype=torch.uint8).expand(1 << 20)), stream=STREAM),
                 lambda: lib.dsn_rotary_axes(ctx, p, r, on(torch.zeros(1, dtype=torch.int32).expand(R)), x, y, stream=STREAM)):
        assert not outcome(lib, ctx, call) and not ctx.seen


def test_descriptor_tensors_lie_on_the_context_s_device(lib):
    i8, f = torch.zeros(C, C, dtype=torch.int8), torch.ones(C)
    x, q, sc, y = (on(torch.zeros(B, R, C, dtype=t)) for t in (torch.bfloat16, torch.int8, torch.float32, torch.bfloat16))
    sc = on(torch.zeros(B, R))
    r, ctx = routing(lib, B), Calls()
    d = lib.make_norm_desc(lib.BF16, R, C, [C], on(f, OnNextGpu))
    l = lib.make_linear_i8_desc(R, C, C, [C], [C], on(i8, OnNextGpu), on(f, OnNextGpu))
    assert not outcome(lib, ctx, lambda: lib.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=sc, stream=STREAM))
    assert not outcome(lib, ctx, lambda: lib.dsn_sliced_linear_i8(ctx, l, r, q, sc, y, stream=STREAM))
    assert not outcome(lib, ctx, lambda: lib.make_linear_i8_desc(R, C, C, [C], [C], on(i8), on(f), bias=on(f, OnNextGpu)))
    assert not ctx.seen
    d = lib.make_norm_desc(lib.BF16, R, C, [C], on(f))
    l = lib.make_linear_i8_desc(R, C, C, [C], [C], on(i8), on(f), bias=on(f))
    assert outcome(lib, ctx, lambda: lib.dsn_rmsnorm_quant(ctx, d, r, x, q=q, scale=sc, stream=STREAM))
    assert outcome(lib, ctx, lambda: lib.dsn_sliced_linear_i8(ctx, l, r, q, sc, y, stream=STREAM))
