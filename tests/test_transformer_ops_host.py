"""8-bit transformer operators on the host: the oracle's forms pinned against independent ones, the binding's checks of
arguments, descriptor layouts and workspace sizes.  No GPU."""
import ctypes
import os

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


def test_oracle_norm_against_library():
    g = np.random.default_rng(1)
    x, res, w = g.normal(size=(3, 5, 24)), g.normal(size=(3, 5, 24)), g.normal(size=24)
    idx, k = [1, 0, 1], [7, 24]
    h, n, scale, steps = O.rmsnorm_quant(x, idx, k, w, 1e-3, res)
    for i, t in enumerate(idx):
        row = torch.from_numpy(x[i, :, :k[t]] + res[i, :, :k[t]])
        ref = torch.nn.functional.rms_norm(row, (k[t],), torch.from_numpy(w[:k[t]]), 1e-3).numpy()
        np.testing.assert_allclose(n[i, :, :k[t]], ref, rtol=1e-12)
        np.testing.assert_allclose(steps[i, :, :k[t]] * scale[i][:, None], ref, rtol=1e-12)
        assert np.allclose(np.max(np.abs(steps[i, :, :k[t]]), axis=-1), 127)
        assert np.all(np.isnan(n[i, :, k[t]:]))
    z = O.rmsnorm_quant(np.zeros((1, 2, 4)), [0], [4])
    assert np.all(z[2] == 0) and np.all(z[3] == 0)


def test_oracle_linear_i8_is_the_sliced_linear_of_the_values():
    g = np.random.default_rng(2)
    x, W = g.integers(-127, 128, size=(4, 3, 20)), g.integers(-127, 128, size=(9, 20))
    sx, sw, b = g.uniform(0.1, 1, (4, 3)), g.uniform(0.1, 1, 9), g.normal(size=9)
    idx, ki, ko = [0, 1, 1, 0], [11, 20], [9, 4]
    got = O.linear_i8(x, sx, W, sw, idx, ki, ko, bias=b, act=O.ACT_GELU)
    ref = O.sliced_linear(x * sx[..., None], W * sw[:, None], idx, ki, ko, bias=b, act=O.ACT_GELU)
    np.testing.assert_allclose(got, ref, rtol=1e-12, atol=1e-12)


def test_oracle_rotary_identities():
    g = np.random.default_rng(3)
    x = g.normal(size=(6, 16))
    pos = g.integers(-50, 50, size=(2, 6))
    y = O.rotary_axes(x, pos, [3, 4])
    np.testing.assert_allclose(O.rotary_axes(y, pos, [3, 4], inverse=True), x, atol=1e-12)       # turning back
    np.testing.assert_array_equal(y[:, 14:], x[:, 14:])                                           # what does not turn
    np.testing.assert_allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))           # lengths stay
    np.testing.assert_array_equal(O.rotary_axes(x, np.zeros((2, 6)), [3, 4]), x)                  # the origin
    # products depend on the difference of positions only
    q, k = g.normal(size=16), g.normal(size=16)
    dots = [O.rotary_axes(q, [p + 5, p + 2], [3, 5], per_axis=True) @ O.rotary_axes(k, [p, p], [3, 5], per_axis=True) for p in (0, 7, 1000)]
    np.testing.assert_allclose(dots, dots[0])
    # interleaved is the halves form on shuffled elements
    sh = np.concatenate([np.arange(0, 16, 2), np.arange(1, 16, 2)])
    np.testing.assert_allclose(O.rotary_axes(x, pos, [3, 5], interleaved=True)[:, sh], O.rotary_axes(x[:, sh], pos, [3, 5]))


def test_descriptor_layouts(lib, tmp_path):
    import subprocess
    names = {"dsn_norm_desc": lib.NormDesc, "dsn_linear_i8_desc": lib.LinearI8Desc, "dsn_rotary_desc": lib.RotaryDesc, "dsn_stats": lib.Stats}
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
            assert got[f"{n}.{f}"] == getattr(cls, f).offset, (n, f)


def test_linear_i8_workspace(lib):
    class W:   # descriptors only hold pointers; nothing is read here
        pass
    d = lib.LinearI8Desc()
    ki, ko = (ctypes.c_int32 * 1)(40), (ctypes.c_int32 * 1)(64)
    d.R, d.C_in, d.C_out, d.ldx, d.ldw, d.ldy, d.T, d.k_in, d.k_out = 7, 40, 64, 48, 48, 64, 1, ki, ko
    d.W, d.w_scale, d.y_dtype = 16, 16, lib.BF16
    assert lib.dsn_linear_i8_workspace_bytes(d, 4000) == 4000 * 7 * 48     # many short samples in input order are gathered
    assert lib.dsn_linear_i8_workspace_bytes(d, 1) == 0 and lib.dsn_linear_i8_workspace_bytes(d, 40) == 0
    d.in_order = lib.GROUPED
    assert lib.dsn_linear_i8_workspace_bytes(d, 4000) == 0
    d.in_order, d.ldw = lib.INPUT_ORDER, 40                                # an invalid descriptor needs nothing: the call refuses it
    assert lib.dsn_linear_i8_workspace_bytes(d, 4000) == 0


def test_binding_refuses_tensors_that_are_not_on_a_gpu(lib):
    f, i8 = torch.zeros(16), torch.zeros(16, 16, dtype=torch.int8)
    for call in (lambda: lib.make_norm_desc(lib.BF16, 1, 16, [16], f), lambda: lib.make_linear_i8_desc(1, 16, 16, [16], [16], i8, f),
                 lambda: lib.make_rotary_desc(lib.BF16, 1, 1, 8, [1], []), lambda: lib.make_rotary_desc(lib.BF16, 1, 1, 8, [1], [1, 1, 1, 1])):
        with pytest.raises(lib.DsnError) as e:
            call()
        assert e.value.code == lib.ERR_INVALID_ARG
