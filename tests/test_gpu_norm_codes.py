"""The codes of the norm, bit for bit against their definition: every fp32 operation rounded once."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, check_status
from transformer_util import groups

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,R,C", [(7, 3, 500), (2000, 1, 96), (2000, 1, 384), (1300, 2, 768), (1300, 1, 1000), (1500, 1, 3000), (1200, 1, 7000),
                                   (2000, 30, 96), (2000, 12, 250), (2000, 8, 384), (1300, 6, 768), (1300, 5, 1000), (1300, 3, 2000)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
def test_codes_are_those_of_the_definition(dsn, B, R, C, name, residual):
    ctx = dsn.Context(0)
    dt = torch.bfloat16 if name == "bf16" else torch.float32
    g = torch.Generator().manual_seed(C + B)
    ld = -(-C // 16) * 16
    x, res = (torch.randn(B, R, ld, generator=g).to(dt) for _ in range(2))
    w = (0.2 + 1.6 * torch.rand(C, generator=g))
    r, _ = groups(dsn, [0] * B, 1)
    q, sc = torch.zeros(B, R, ld, dtype=torch.int8, device=DEV), torch.zeros(B, R, device=DEV)
    d = dsn.make_norm_desc(dsn.BF16 if name == "bf16" else dsn.F32, R, C, [C], w.to(DEV), ldx=ld, ld_res=ld, ldq=ld)
    dsn.dsn_rmsnorm_quant(ctx, d, r, x.to(DEV), q=q, scale=sc, residual=res.to(DEV) if residual else None)
    check_status(ctx, dsn)
    # numpy's fp32 operations round once each
    h = x.float().numpy()[..., :C]
    if residual:
        h = h + res.float().numpy()[..., :C]
    v = h * w.numpy()
    inv = np.float32(127) * (np.float32(1) / np.max(np.abs(v), axis=-1, keepdims=True))
    want = np.rint(v * inv)
    assert v.dtype == want.dtype == np.float32
    np.testing.assert_array_equal(q.cpu().numpy()[..., :C], want)
