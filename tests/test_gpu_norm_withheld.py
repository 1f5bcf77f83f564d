"""The streaming form of the norm when a row never arrives: the wait gives up, the status says so, and the stream, which is written in place, holds
old or new values and nothing else.  Nothing faults: the copy of one row is left out, its barrier never completes, every wait is bounded."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
TIMEOUT = -7
WAIT_US = 4                                                       # word of the status block with the limit of a wait
MARK = 77


@pytest.fixture(scope="module")
def withheld(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("withheld") / "libnorm_withheld.so")
    csrc = os.path.join(ROOT, "paper_2109_10060_b200", "csrc")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-shared", "-cudart", "shared", "-Xcompiler", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(HERE, "norm_withheld.cu"), "-o", out], check=True)
    fn = ctypes.CDLL(out).norm_withheld
    vp, i32 = ctypes.c_void_p, ctypes.c_int
    fn.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp]
    return fn


# widths for 16, 32, 64, 128 and 256 threads a row
@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("k", [120, 380, 1000, 2040, 4090, 8000])
@pytest.mark.parametrize("codes", [True, False])
def test_a_row_that_never_arrives_leaves_the_stream_as_it_was(withheld, name, k, codes):
    dt = torch.bfloat16 if name == "bf16" else torch.float32
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows, ld = max(16 * sms, -(-(5 << 20) // k)) + 3, -(-k // 16) * 16
    g = torch.Generator(device=DEV).manual_seed(k)
    x, res = (torch.randn(rows, ld, generator=g, device=DEV).to(dt) for _ in range(2))
    offsets, perm = torch.tensor([0, rows], dtype=torch.int32, device=DEV), torch.arange(rows, dtype=torch.int32, device=DEV)
    new = (x.float() + res.float()).to(dt)
    for row in (5, rows // 2):                                    # asked for before anything has arrived; into a slot that held another row
        for which in (x, res):
            sm = x.clone()
            src = sm if which is x else res
            q, sc = torch.full((rows, ld), MARK, dtype=torch.int8, device=DEV), torch.full((rows,), float(MARK), device=DEV)
            status = torch.zeros(8, dtype=torch.int32, device=DEV)
            status[WAIT_US] = 1000
            at = src.data_ptr() + row * ld * src.element_size()
            torch.cuda.synchronize()
            err = withheld(sm.data_ptr(), res.data_ptr(), q.data_ptr() if codes else None, sc.data_ptr() if codes else None, rows, k, ld, int(name == "f32"),
                           at, at + 16, offsets.data_ptr(), perm.data_ptr(), status.data_ptr(), sms, None)
            assert err == 0
            torch.cuda.synchronize()
            assert status[0].item() == TIMEOUT
            assert torch.equal(sm[row], x[row])                   # the row that did not come
            assert bool(((sm == x) | (sm == new))[:, :k].all())
            assert torch.equal(sm[:, k:], x[:, k:])
            if codes:
                assert bool((q[row] == MARK).all()) and sc[row].item() == MARK
                done = sc != MARK                                 # rows with a scale are finished
                assert bool((sm == new)[done, :k].all()) and bool((q[~done] == MARK).all())
    # and with nothing withheld, every row comes
    sm, status = x.clone(), torch.zeros(8, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    assert withheld(sm.data_ptr(), res.data_ptr(), None, None, rows, k, ld, int(name == "f32"), None, None, offsets.data_ptr(), perm.data_ptr(),
                    status.data_ptr(), sms, None) == 0
    torch.cuda.synchronize()
    assert status[0].item() == 0 and torch.equal(sm[:, :k], new[:, :k])
