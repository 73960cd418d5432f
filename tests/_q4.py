"""The 4-bit cache in numpy, 64 bits, from its definition in include/wm.h, and small
paged caches in that form for the tests of its calls."""
from __future__ import annotations

import numpy as np
import torch

from paper_2608_18486_gb300.session import Q4Cache
from tests._longctx import Cache

MAGS = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
SCALES = (np.arange(227, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)  # by byte


def nearest(x, grid):
    """Index of the nearest of an ascending grid (last axis of grid), ties to the even one.
    Comparisons with (g_i + g_i+1) / 2, which is exact in 64 bits."""
    mid = (grid[..., 1:] + grid[..., :-1]) / 2
    odd = np.arange(mid.shape[-1]) % 2 == 1  # a tie between odd i and i + 1 goes up
    return ((x[..., None] > mid) | ((x[..., None] == mid) & odd)).sum(-1)


def quantise(x):
    """Codes [..., d] and scale bytes [..., d / 16] (uint8) of float64 rows."""
    g = x.reshape(*x.shape[:-1], -1, 16)
    top = np.abs(g).max(-1)
    bad = ~np.isfinite(g).all(-1)
    byte = nearest(np.where(bad, 0, top), 6 * SCALES)
    s = SCALES[byte][..., None]
    code = nearest(np.where(bad[..., None], 0, np.abs(g)), MAGS * s[..., None]) + 8 * np.signbit(g)
    code = np.where((s == 0) | bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def values(code, byte):
    s = (byte.astype(np.uint16) << 7).view(np.float16).astype(np.float64)
    v = np.where(code >= 8, -MAGS[code & 7], MAGS[code & 7])
    return (v.reshape(*code.shape[:-1], -1, 16) * s[..., None]).reshape(code.shape)


def tile_shape(P, d):
    n = min(P, 16)
    return n, (n * (d + d // 8) + 15) // 16 * 16


def pool_view(buf, k, pages, Hkv, P, d):
    n, size = tile_shape(P, d)
    return buf[:k * pages * Hkv * (P // n) * size].reshape(k, pages, Hkv, P // n, size)


def put_row(pool, c, page, h, slot, X, code, byte):
    """Row of slot (in page) into pool [k][pages][Hkv][P / n][tile]."""
    d = code.shape[-1]
    n = tile_shape_of(pool, d)
    r, t = slot % n, pool[c, page, h, slot // n]
    t[(X * n + r) * (d // 2):][:d // 2] = code[0::2] | code[1::2] << 4
    t[n * d + (X * n + r) * (d // 16):][:d // 16] = byte


def tile_shape_of(pool, d):
    return min(16, pool.shape[-1] // (d + d // 8))


class Q4(Cache):
    """A Cache whose rows are also held in 4 bits, in pages of their own (q4_table).
    Everything that no slot < lens reaches is 0xFF: NaN scales."""

    def __init__(self, lens, **kw):
        super().__init__(lens, **kw)
        self.source = self.kd, self.vd
        self.q4_pages = self.num_pages + 2
        order = self.rng.permutation(self.q4_pages)
        self.q4_table = np.where(self.table >= 0, order[np.clip(self.table, 0, None)], -5).astype(np.int32)
        n, size = tile_shape(self.P, self.d)
        self.pool = np.full((self.k, self.q4_pages, self.Hkv, self.P // n, size), 0xFF, dtype=np.uint8)
        self.kd, self.vd = (np.full_like(x, np.nan) for x in self.source)
        for x, (src, to) in enumerate(zip(self.source, (self.kd, self.vd))):
            fill = ~np.isnan(src[..., 0])
            code, byte = quantise(np.where(fill[..., None], src, 0))
            to[fill] = values(code, byte)[fill]
            for c, pg, h, s in zip(*np.nonzero(fill)):
                put_row(self.pool, c, order[pg], h, s, x, code[c, pg, h, s], byte[c, pg, h, s])

    def q4(self):
        q4 = Q4Cache(self.session_cfg(), self.q4_pages)
        q4.cache_buf[:self.pool.size] = torch.from_numpy(self.pool.reshape(-1)).cuda()
        return q4

    def session_cfg(self):
        from paper_2608_18486_gb300 import _lib as W
        return W.make_config(self.k, self.k, 64, self.Hq, self.Hkv, self.d, 1, self.P, self.dtype, list(range(self.k)))

    def q4_dev(self):
        return torch.from_numpy(self.q4_table).cuda(), torch.from_numpy(self.lens).cuda()

    def bound(self, c, b, hq, q, ts, steps):
        """(exact output, largest error of an element) of one query row over slots ts.

        A matrix instruction adds 17 terms, each cut below 2^-23 of the largest: at most 17 *
        2^-23 of a block's largest |q k|, one block (three instructions in fp32) per 16
        features; scaling and the exponent's argument round a few times more.  A weight
        is off by 2 ds for that, its parts by 2^-11 (fp16) or 2^-22 (two of them), and the
        sums of a warp's `steps` products by 17 * 2^-23 each (fp32: 34 in all, since
        every step's own products are added with rounding).  The result is
        rounded by 2^-8 (bf16) or 2^-24 of itself."""
        want, p, _, vmax = self.attend(c, b, hq, q, ts)
        if len(ts) == 0:
            return want, 0.0
        K = self.rows(self.kd, c, b, hq // self.G, ts)
        ds = (110 + self.d) * 2.0 ** -24 * float((np.abs(K) @ np.abs(q)).max()) / np.sqrt(self.d)
        if self.dtype == "bf16":
            rel = 2 * ds + 2.0 ** -11 + steps * 17 * 2.0 ** -23 + 64 * 2.0 ** -24
            return want, rel * vmax + 2.0 ** -8 * float(np.abs(want).max())
        return want, (2 * ds + 2.0 ** -22 + 34 * 2.0 ** -23 + 64 * 2.0 ** -24) * vmax
