"""The norm at the ends of what fp32 holds: weights and rows so small or large that their squares or products leave the range, against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV, check_status
from transformer_util import U, groups, half_step, rows_with_pitch, values

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
LEAST = {"bf16": 2.0 ** -133, "f32": 2.0 ** -149}                 # smallest positive values


@pytest.fixture(scope="module")
def ctx(dsn):
    return dsn.Context(0)


def run(dsn, ctx, x, w, name, eps, raw):
    """x [rows][C] in fp32 values, one row a sample."""
    B, C = x.shape
    ld = -(-C // 16) * 16
    r, _ = groups(dsn, [0] * B, 1)
    xd = rows_with_pitch(x[:, None], ld, DT[name], 1e30)
    q, sc = torch.full((B, ld), 99, dtype=torch.int8, device=DEV), torch.zeros(B, device=DEV)
    y = torch.zeros(B, ld, dtype=DT[name], device=DEV)
    wd = None if w is None else torch.from_numpy(w.astype(np.float32)).to(DEV)
    d = dsn.make_norm_desc(dsn.BF16 if name == "bf16" else dsn.F32, 1, C, [C], wd, eps=eps, ldx=ld, ldq=ld, ldy=ld)
    dsn.dsn_rmsnorm_quant(ctx, d, r, xd, q=None if raw else q, scale=None if raw else sc, y=y)
    check_status(ctx, dsn)
    return values(q)[:, :C], values(sc), values(y)[:, :C]


def check(dsn, ctx, x, w, name, eps=1e-6):
    hs, least = half_step(DT[name]), LEAST[name]
    _, n, scale, steps = (a[:, 0] for a in O.rmsnorm_quant(x[:, None], [0] * len(x), [x.shape[1]], w, eps))
    assert np.all(np.abs(n) < 3.3e38)
    q, sc, y = run(dsn, ctx, x, w, name, eps, False)
    # as for rows of ordinary size; a scale below 2^-126 is rounded to a multiple of 2^-149, twice
    assert np.all(np.abs(q - steps) <= 0.5 + 127 * 7 * U)
    assert np.all(np.abs(sc - scale) <= 48 * U * scale + 2.0 ** -149)
    ref = q * sc[:, None]
    assert np.all(np.abs(y - ref) <= (hs + 2 * U) * np.abs(ref) + least)
    _, _, y = run(dsn, ctx, x, w, name, eps, True)
    # (a product that is below 2^-126 before the root's factor, up to 1e10, keeps 2^-150 times it; the range below is chosen so that it does not)
    assert np.all(np.abs(y - n) <= (hs + 48 * U) * np.abs(n) + least)


# a row for few and one for many threads, rows enough for the streaming form and not
SHAPES = [(7, 200), (2, 1100), (1300, 96 * 48), (45000, 128)]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SHAPES)
@pytest.mark.parametrize("size", [1e-44, 1e-39, 2e-38, 3e-37, 1e-30, 1e30, 3e37, 1.5e38])
def test_weights_of_any_size(dsn, ctx, name, rows, C, size):
    g = np.random.default_rng(C)
    x = torch.from_numpy(g.uniform(0.5, 1, (rows, C)) * g.choice([-1, 1], (rows, C))).to(DT[name]).double().numpy()
    x[1 % rows] = 0
    w = (size * g.uniform(0.5, 1, C) * g.choice([-1, 1], C)).astype(np.float32).astype(np.float64)
    if size < 1e-36:
        x[3 % rows] *= 2.0 ** 20
    check(dsn, ctx, x, w, name)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_rows_of_any_size(dsn, ctx, name, rows, C):
    """Every row another power of two, from the smallest normal values (eps decides) to the largest."""
    g = np.random.default_rng(rows)
    e = np.resize(np.arange(-125, 127), rows)
    x = torch.from_numpy(g.uniform(0.5, 1, (rows, C)) * g.choice([-1, 1], (rows, C))).to(DT[name]).double().numpy() * 2.0 ** e[:, None]
    w = g.uniform(0.5, 2, C).astype(np.float32).astype(np.float64)
    for eps in (1e-20, 1e-6):
        check(dsn, ctx, x, w, name, float(np.float32(eps)))
        check(dsn, ctx, x, None, name, float(np.float32(eps)))


@pytest.mark.parametrize("rows,C", SHAPES)
def test_rows_and_weights_of_opposite_size(dsn, ctx, rows, C):
    g = np.random.default_rng(rows)
    x = torch.from_numpy(g.uniform(0.5, 1, (rows, C))).float().double().numpy()
    for ex, ew in ((100, -140), (-60, 120), (60, 100), (120, 126), (-100, -30)):
        w = np.float32(g.uniform(0.5, 1, C)).astype(np.float64) * 2.0 ** ew
        w = w.astype(np.float32).astype(np.float64)
        check(dsn, ctx, x * 2.0 ** ex, w, "f32", float(np.float32(1e-20)))
