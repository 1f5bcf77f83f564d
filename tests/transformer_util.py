"""Helpers of the tests of the 8-bit transformer operators."""
import numpy as np
import torch

from gpu_util import DEV

U = 2.0 ** -24                       # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def groups(dsn, idx, T):
    """Routing arrays of a batch, built on the host; also the stable grouped order."""
    idx = np.asarray(idx, dtype=np.int64)
    B = len(idx)
    perm = np.argsort(idx, kind="stable")
    inv = np.empty(B, np.int64)
    inv[perm] = np.arange(B)
    counts = np.bincount(idx, minlength=T)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)
    dummy = lambda a: up(a) if len(a) else torch.zeros(1, dtype=torch.int32, device=DEV)
    return dsn.make_routing(B, T, up(counts), up(offsets), dummy(perm), dummy(inv)), perm


def rows_with_pitch(a, ld, dtype, fill):
    """[B][R][C] values -> device [B][R][ld] of `dtype`, the columns beyond C filled with `fill`."""
    t = torch.full((*a.shape[:2], ld), fill, dtype=dtype)
    t[..., :a.shape[2]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t.to(DEV)


def values(t):
    return t.detach().cpu().double().numpy()
