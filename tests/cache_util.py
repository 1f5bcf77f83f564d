"""Helpers of the tests of the 4-bit cache."""
import numpy as np
import torch

from oracle import dsn_oracle as O
from gpu_util import DEV

U = 2.0 ** -8      # half a step of bf16, relative


def up(a, dt=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(DEV)


class Pages:
    """Pages of a cache on the host: random codes and pairs everywhere, tokens by request through a shuffled table.  What no token of a request
    uses (the rest of its last page, pages nobody holds) is filled with NaN pairs."""

    def __init__(self, g, lengths, H, D, page, spare=2, k_gain=1.0):
        self.H, self.D, self.page, n = H, D, page, D // 64
        self.lengths = list(lengths)
        count = [-(-L // page) for L in lengths]
        self.n_pages, self.max_pages = sum(count) + spare, max(max(count), 1)
        order = g.permutation(self.n_pages)
        self.table = np.full((len(count), self.max_pages), -1, np.int32)
        at = 0
        for i, c in enumerate(count):
            self.table[i, :c] = order[at:at + c]
            at += c
        tokens = (self.n_pages, H, page)
        self.code = g.integers(0, 16, size=(*tokens, 2, n, 64)).astype(np.uint8)
        self.s = O.round_bf16(g.uniform(0.1, 0.4, size=(*tokens, 2, n)))
        self.z = O.round_bf16(0.3 * g.normal(size=(*tokens, 2, n)))
        self.s[:, :, :, 0] = O.round_bf16(self.s[:, :, :, 0] * k_gain)
        used = np.zeros((self.n_pages, page), bool)
        for i, L in enumerate(lengths):
            for t in range(L):
                used[self.table[i, t // page], t % page] = True
        dead = ~used
        self.s = np.where(dead[:, None, :, None, None], np.nan, self.s)
        self.z = np.where(dead[:, None, :, None, None], np.nan, self.z)

    def bytes(self):
        """[n_pages][H][page / 16][18 D]"""
        P, H, page, n = self.n_pages, self.H, self.page, self.D // 64
        parts = []
        for half in range(2):
            c = self.code[:, :, :, half]                                        # [P, H, page, n, 64]
            c = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(P, H, page // 16, 16, n, 32).transpose(0, 1, 2, 4, 3, 5)
            pr = np.stack([self.s[:, :, :, half], self.z[:, :, :, half]], -1)
            bits = (np.ascontiguousarray(pr, np.float32).view(np.uint32) >> 16).astype(np.uint16)
            bits = np.ascontiguousarray(bits).view(np.uint8).reshape(P, H, page // 16, 16, n, 4).transpose(0, 1, 2, 4, 3, 5)
            parts += [c.reshape(P, H, page // 16, -1), bits.reshape(P, H, page // 16, -1)]
        return np.concatenate(parts, -1)

    def kv(self, i, head):
        """Keys and values of request i in a head, [L][D] each."""
        t = np.arange(self.lengths[i])
        pg, at = self.table[i, t // self.page], t % self.page
        return [O.cache_values(self.code[pg, head, at, half], self.s[pg, head, at, half], self.z[pg, head, at, half]) for half in range(2)]


    def v_size(self, i, head):
        """|middle| + |scale (code - 8)| of the values of request i in a head, [L][D]."""
        t = np.arange(self.lengths[i])
        pg, at = self.table[i, t // self.page], t % self.page
        code, s, z = self.code[pg, head, at, 1], self.s[pg, head, at, 1], self.z[pg, head, at, 1]
        return O.cache_values(np.abs(code.astype(np.float64) - 8) + 8, s, np.abs(z))


def attention_bound(q, k, v_size, p, out, scale):
    """How far an output may be off, element by element.

    Rounding the output moves it by U |out|.  Rounding a probability (times a scale) and a value to bf16 before the second product moves a term by 2 U of
    its size.  A value is middle + scale (code - 8), and a kernel may sum the two parts apart: p middle, and round(p scale) (code - 8) with
    |round(p scale) - p scale| <= U p scale.  The parts can cancel (a value can be exactly 0), the roundings do not, so a term's size is
    p (|middle| + |scale (code - 8)|), which is what v_size holds; fp32 sums of the parts add 2^-12 of the same.  A kernel that rounds the key elements to bf16 moves a score by at most U sum |q_d k_d| |scale|; sums in fp32 add a share of 2^-12 of
    that.  A score off by e moves every weight by a factor within exp(2 e), numerator and denominator together."""
    size = abs(scale) * (np.abs(q) @ np.abs(k).T)                               # [n][L]; a movement has no sign
    e = (U + 2.0 ** -12) * np.where(p > 0, size, 0.0).max(-1, keepdims=True) if p.shape[1] else np.zeros((len(q), 1))
    terms = p @ v_size if p.shape[1] else 0.0
    return U * np.abs(out) + (2 * U + 2.0 ** -12 + np.expm1(2 * e)) * terms + 1e-30


def make_desc(dsn, pages, R, heads, group, **kw):
    return dsn.make_cache_desc(R, pages.H, pages.D, heads, group=group, page=pages.page, n_pages=pages.n_pages, max_pages=pages.max_pages, **kw)


def workspace(dsn, d, B):
    n = dsn.dsn_cache_attention_q4_workspace_bytes(d, B)
    return torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) if n else None
