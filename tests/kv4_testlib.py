"""The 4-bit cache's format in 64 bits on the CPU, and caches for the tests (shared by the tests of the cache's calls)."""
from __future__ import annotations

import numpy as np
import torch


def quantise64(x: np.ndarray, group: int):
    """Scale, zero point and codes of [..., D] by the format's definition, in binary64."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, group))
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    lo, hi = np.minimum(g.min(-1), 0.0), np.maximum(g.max(-1), 0.0)
    m, e = np.frexp((hi - lo) / 15)
    e = np.maximum(e, -125)
    s = np.ldexp(np.rint(np.ldexp((hi - lo) / 15, 20 - e)), e - 20)
    d = np.where(s > 0, s, 1.0)
    zero = np.where(s > 0, np.clip(np.rint(-lo / d), 0, 15), 0.0)
    q = np.where(s[..., None] > 0, np.clip(np.rint(g / d[..., None]) + zero[..., None], 0, 15), 0.0)
    return np.where(bad, np.nan, s), zero, q


def stored64(x, group: int) -> np.ndarray:
    """What the cache stands for."""
    x = x.double().cpu().numpy() if isinstance(x, torch.Tensor) else x
    s, zero, q = quantise64(x, group)
    return (s[..., None] * (q - zero[..., None])).reshape(x.shape)


class Cache:
    """A cache on the GPU with scattered pages, guard bytes around the pool and 0xA5 in it, and the same content in 64 bits."""

    def __init__(self, lens, page=64, heads=2, D=128, group=64, dt=torch.bfloat16, room=None, extra=3, seed=0, layers=1, layer=0):
        import paper_2412_07174_b200 as scap
        self.scap, self.page, self.heads, self.D, self.group, self.dt = scap, page, heads, D, group, dt
        rng = np.random.default_rng(seed)
        room = room or max(max(lens), 1)
        self.width = -(-room // page)
        B = len(lens)
        n = B * self.width + extra
        ids = rng.permutation(n)[:B * self.width].reshape(B, self.width)
        self.bytes = scap.scap_kv4_page_bytes(page, heads, D, group)
        self.raw = torch.full((n + 2, layers * self.bytes), 0xA5, dtype=torch.uint8, device="cuda")
        self.pool = self.raw[1:-1]
        self.table = torch.tensor(ids, dtype=torch.int32, device="cuda")
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.view = self.pool[:, layer * self.bytes:(layer + 1) * self.bytes]
        self.cache = scap.ScapKv4(self.view, page, heads, D, group, self.table, self.lens)
        self.k = [np.zeros((0, heads, D)) for _ in lens]
        self.v = [np.zeros((0, heads, D)) for _ in lens]

    def guards_intact(self):
        return bool((self.raw[0] == 0xA5).all()) and bool((self.raw[-1] == 0xA5).all())


def starts(counts):
    return torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")


def tokens(n, heads, D, dt, seed):
    """Values with outlier channels, means off zero and different sizes per token."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, heads, D, generator=g, device="cuda") * torch.exp(torch.randn(heads, D, generator=g, device="cuda"))
    x = x * torch.exp(2 * torch.randn(n, heads, 1, generator=g, device="cuda")) + 0.3 * torch.randn(heads, D, generator=g, device="cuda")
    return x.to(dt)
