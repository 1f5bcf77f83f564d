"""The many-rows attention over the 4-bit cache when a tile never arrives: the waits give up, the status says so, and before its CTA ends the loader
waits for every copy that it issued, those of the missing tile among them, and both issuing warps for their products.  Nothing faults: one page's copies are left out, every wait is bounded."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from cache_util import Pages, up
from gpu_util import DEV

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
TIMEOUT = -7
WAIT_US = 4                                                       # word of the status block with the limit of a wait


@pytest.fixture(scope="module")
def withheld(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("withheld") / "libcache_withheld.so")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-shared", "-cudart", "shared", "-Xcompiler", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2109_10060_b200", "csrc"),
                    os.path.join(HERE, "cache_rows_withheld.cu"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    vp, i32 = ctypes.c_void_p, ctypes.c_int
    lib.cache_rows_withheld.argtypes = [vp] * 7 + [i32] * 2 + [vp] * 3 + [i32] + [vp] * 3
    lib.cache_rows_ws_bytes.restype = ctypes.c_long
    return lib


@pytest.mark.parametrize("tile", [0, 1, 2, 4])
def test_a_tile_that_never_arrives(withheld, tile):
    """148 CTAs of five tiles each; tile number `tile` of the tenth is left out."""
    g = np.random.default_rng(tile)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    ctas = min(sms, 148)
    rows, L = 40, 64 * 5 * ctas
    pages = Pages(g, [L], 1, 64, 64)
    raw, table, lengths = torch.from_numpy(pages.bytes()).to(DEV), up(pages.table), up([L])
    offsets, perm = up([0, 1]), up([0])
    x = torch.randn(1, rows, 192, device=DEV).to(torch.bfloat16)
    out = torch.zeros(1, rows, 64, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((withheld.cache_rows_ws_bytes(),), 0xff, dtype=torch.uint8, device=DEV)
    status = torch.zeros(8, dtype=torch.int32, device=DEV)
    status[WAIT_US] = 1000
    per = raw.numel() // pages.n_pages
    at = raw.data_ptr() + int(pages.table[0, 5 * 9 + tile]) * per
    drain, ended = np.zeros((148, 2), np.int32), np.zeros(148, np.int32)

    def go(first, last):
        torch.cuda.synchronize()
        err = withheld.cache_rows_withheld(x.data_ptr(), out.data_ptr(), raw.data_ptr(), table.data_ptr(), lengths.data_ptr(), offsets.data_ptr(), perm.data_ptr(), rows,
                                           pages.n_pages, first, last, status.data_ptr(), sms, ws.data_ptr(), drain.ctypes.data,
                                           ended.ctypes.data)
        assert err == 0

    go(0, 0)
    assert status[0].item() == 0 and np.all(drain == -1) and not ended.any()
    whole = out.clone()
    go(at, at + per)
    assert status[0].item() == TIMEOUT
    assert np.all(np.delete(drain, 9, 0) == -1)
    first, asked = drain[9]
    assert asked == tile + 1 and first == max(0, asked - 2)
    assert ended[9] in (1, 2) and not np.delete(ended, 9).any()      # the half without rows may have had nothing left to wait for
    status[0] = 0
    go(0, 0)
    assert status[0].item() == 0 and torch.equal(out, whole) and bool(out.isfinite().all())
