"""GELU of pre-activations far from zero, in every kernel that has it: x/2 (1 + erf(x / sqrt 2)) is x or nothing there.  Weights of zeros and ones hand
the inputs to the activation as they are."""
import os

import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV, check_status
from transformer_util import groups, half_step, values

pytestmark = pytest.mark.gpu
C = 64


def inputs(B, R):
    """[B][R][C] values that bf16 represents: a fine grid over -40 .. 40, the places where the fitted quintic turns round and changes sign, and far ones."""
    far = np.array([1e2, 1e4, 1e9, 1e18, 1e19, 2e19, 1e30, 3e38])
    edge = np.array([5.875, 6, 8.25, 8.3125, 10.125, 10.1875, 10.25, 11, 11.0625, 12, 16, 20])
    v = np.concatenate([edge, -edge, far, -far, np.linspace(-40, 40, 1501)])
    x = np.resize(v, B * R * C).reshape(B, R, C)
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def check(got, x, dt=torch.bfloat16, fitted=True, stored_again=False):
    z = np.clip(x, -60, 60)                                       # (beyond, the oracle's erf is +-1 long since)
    ref = np.where(np.abs(x) > 60, np.maximum(x, 0), O.activation(z, O.ACT_GELU))
    # the hardware tanh is within 2^-11 of its value, half of |x| times that; the fit within 3e-5 of erf's GELU; one rounding at the end.  Formula
    # 7.1.26: erf within 1.5e-7, half of |x| times that, and a few roundings of |x|; CUDA's erff: the same few roundings
    tol = np.abs(x) * 2.0 ** -12 + 3e-5 if fitted else np.abs(x) * (0.75e-7 + 8 * 2.0 ** -24)
    tol = tol + half_step(dt) * (2 if stored_again else 1) * np.abs(ref)
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - ref) <= tol), (float(x[np.abs(got - ref) > tol].flat[0]), float(got[np.abs(got - ref) > tol].flat[0]))


def context(dsn, **switches):
    old = {k: os.environ.get(k) for k in switches}
    os.environ.update(switches)
    try:
        return dsn.Context(0)
    finally:
        for k, v in old.items():
            os.environ.pop(k) if v is None else os.environ.__setitem__(k, v)


def up(x):
    return torch.from_numpy(x).to(torch.bfloat16).to(DEV)


def eye():
    return torch.eye(C, dtype=torch.bfloat16, device=DEV)


@pytest.mark.parametrize("mode", ["pair", "1cta"])
@pytest.mark.parametrize("form", ["plain", "bias", "residual"])
@pytest.mark.parametrize("grouped", [False, True])
def test_gelu_of_the_bf16_linear_layer(dsn, mode, form, grouped):
    ctx = context(dsn, DSN_GEMM_MODE=mode)
    B, R = 6, 50
    x = inputs(B, R)
    r, _ = groups(dsn, [0] * B, 1)
    zero = torch.zeros(B, R, C, dtype=torch.bfloat16, device=DEV)
    d = dsn.make_linear_desc(dsn.BF16, R, C, C, [C], [C], eye(), bias=torch.zeros(C, device=DEV) if form == "bias" else None, act=dsn.ACT_GELU,
                             residual=zero if form == "residual" else None, in_order=int(grouped), out_order=int(grouped))
    y = torch.zeros_like(zero)
    dsn.dsn_sliced_linear(ctx, d, r, up(x), y)
    check_status(ctx, dsn)
    st = ctx.stats()
    assert st["launches_gemm_pair" if mode == "pair" else "launches_gemm_one_cta"] == 1
    check(values(y), x)


@pytest.mark.parametrize("bias", [False, True])
def test_gelu_of_the_3x3_layer(dsn, bias):
    ctx = dsn.Context(0)
    B, H = 4, 14
    x = inputs(B, H * H)
    r, _ = groups(dsn, [0] * B, 1)
    W = torch.zeros(C, 3, 3, C, dtype=torch.bfloat16, device=DEV)
    W[:, 1, 1] = eye()
    y = torch.zeros(B, H * H, C, dtype=torch.bfloat16, device=DEV)
    d = dsn.make_conv_desc(dsn.BF16, H, H, 3, 1, C, C, [C], [C], W, bias=torch.zeros(C, device=DEV) if bias else None, act=dsn.ACT_GELU)
    # (3e38 times the zeros of the other taps is 0)
    dsn.dsn_sliced_conv(ctx, d, r, up(x), y)
    check_status(ctx, dsn)
    assert ctx.stats()["launches_gemm_halo"] == 1
    check(values(y), x)


def test_gelu_of_a_chain(dsn):
    ctx = dsn.Context(0)
    B, R = 5, 196
    x = inputs(B, R)
    layers = [dsn.make_linear_desc(dsn.BF16, R, C, C, [C], [C], eye(), act=dsn.ACT_GELU), dsn.make_linear_desc(dsn.BF16, R, C, C, [C], [C], eye())]
    L = dsn.make_layer_desc(B, 1, layers)
    ws = torch.empty(dsn.dsn_layer_workspace_bytes(L), dtype=torch.uint8, device=DEV)
    y = torch.zeros(B, R, C, dtype=torch.bfloat16, device=DEV)
    dsn.dsn_layer_forward(ctx, L, up(x), torch.zeros(B, dtype=torch.int32, device=DEV), y, ws)
    check_status(ctx, dsn)
    assert ctx.stats()["launches_gemm_chain"] == 1
    check(values(y), x, stored_again=True)


@pytest.mark.parametrize("fused", [False, True])
def test_gelu_of_the_separable_block(dsn, fused):
    ctx = context(dsn, DSN_DWPW="fused" if fused else "0")
    B, H = 4, 14
    x = inputs(B, H * H)
    Wdw = torch.zeros(3, 3, C, dtype=torch.bfloat16, device=DEV)
    Wdw[1, 1] = 1
    dw = dsn.make_depthwise_desc(H, H, 3, 1, C, [C], [3], Wdw, act=dsn.ACT_GELU)
    pw = dsn.make_conv_desc(dsn.BF16, H, H, 1, 0, C, C, [C], [C], eye())
    L = dsn.make_layer_desc(B, 1, [dw, pw])
    ws = torch.empty(dsn.dsn_layer_workspace_bytes(L), dtype=torch.uint8, device=DEV)
    y = torch.zeros(B, H * H, C, dtype=torch.bfloat16, device=DEV)
    dsn.dsn_layer_forward(ctx, L, up(x), torch.zeros(B, dtype=torch.int32, device=DEV), y, ws)
    check_status(ctx, dsn)
    assert ctx.stats()["launches_dwpw"] == int(fused)
    check(values(y), x, stored_again=True)


@pytest.mark.parametrize("y_type", ["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 32, 33, 300])
@pytest.mark.parametrize("residual", [False, True])
def test_gelu_of_the_8_bit_linear_layer(dsn, y_type, B, residual):
    """Few rows and many: the same function, whichever kernel runs."""
    ctx = dsn.Context(0)
    g = np.random.default_rng(B)
    dt = torch.bfloat16 if y_type == "bf16" else torch.float32
    q = g.integers(-127, 128, size=(B, 1, C))
    q[..., :4] = [127, -127, 40, -40]
    s = g.choice([2.0 ** -5, 0.3125, 2.0 ** 60], size=(B, 1))   # few digits: the products are exact in fp32
    s[0] = 0.3125
    r, _ = groups(dsn, [0] * B, 1)
    f = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV)
    y = torch.zeros(B, 1, C, dtype=dt, device=DEV)
    d = dsn.make_linear_i8_desc(1, C, C, [C], [C], torch.eye(C, dtype=torch.int8, device=DEV), torch.ones(C, device=DEV), act=dsn.ACT_GELU,
                                residual=torch.zeros_like(y) if residual else None, y_dtype=dsn.BF16 if y_type == "bf16" else dsn.F32)
    dsn.dsn_sliced_linear_i8(ctx, d, r, torch.from_numpy(q.astype(np.int8)).to(DEV), f(s), y)
    check_status(ctx, dsn)
    check(values(y), q * s[..., None], dt, fitted=y_type == "bf16")


@pytest.mark.parametrize("B", [3, 40])
def test_gelu_of_the_fp32_linear_layer(dsn, B):
    ctx = dsn.Context(0)
    x = inputs(B, 7)
    r, _ = groups(dsn, [0] * B, 1)
    y = torch.zeros(B, 7, C, device=DEV)
    dsn.dsn_sliced_linear(ctx, dsn.make_linear_desc(dsn.F32, 7, C, C, [C], [C], torch.eye(C, device=DEV), act=dsn.ACT_GELU), r,
                          torch.from_numpy(x.astype(np.float32)).to(DEV), y)
    check_status(ctx, dsn)
    check(values(y), x, torch.float32, fitted=False)
