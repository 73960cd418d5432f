"""Small paged caches with 64-bit references for the long-context operators.

Pools start as NaN everywhere and only the slots a test makes visible get
values, so anything read from a masked slot shows.  References are numpy
float64, written from the operators' definitions.
"""
from __future__ import annotations

import numpy as np
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import DecodeSession


class Cache:
    """B sequences of ``lens`` slots; K, V [k][B][Hkv][T][d] float64 (the
    stored values), NaN where nothing was written."""

    def __init__(self, lens, *, Hkv, G, d, page, dtype="bf16", k=2, shared=0, seed=0, extra_pages=3,
                 max_pages=None, visible=None):
        self.lens = np.asarray(lens, dtype=np.int32)
        self.B, self.Hkv, self.G, self.Hq, self.d, self.P = len(lens), Hkv, G, Hkv * G, d, page
        self.k, self.dtype = k, dtype
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.max_pages = max_pages or max(max(int(n) for n in lens) // page, shared) + 2
        T = self.max_pages * page
        need = [max(-(-int(n) // page), shared) for n in lens]
        self.num_pages = shared + sum(n - shared for n in need) + extra_pages
        order = rng.permutation(self.num_pages).astype(np.int32)
        self.table = np.full((self.B, self.max_pages), -7, dtype=np.int32)
        self.table[:, :shared] = order[:shared]
        at = shared
        for b in range(self.B):
            self.table[b, shared:need[b]] = order[at:at + need[b] - shared]
            at += need[b] - shared
        tdt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.tdt = tdt
        shape = (k, self.num_pages, Hkv, page, d)
        kp, vp = torch.full(shape, float("nan"), dtype=tdt), torch.full(shape, float("nan"), dtype=tdt)
        # visible(b): the slots of sequence b that hold values (default: all)
        for b in range(self.B):
            ts = np.asarray(list(range(int(self.lens[b])) if visible is None else visible(b)), dtype=np.int64)
            if shared and len(ts):  # slots of the shared pages are written once
                first = torch.from_numpy(self.table[b, ts // page].astype(np.int64)), torch.from_numpy(ts % page)
                ts = ts[torch.isnan(kp[0, first[0], 0, first[1], 0]).numpy()]
            at = torch.from_numpy(self.table[b, ts // page].astype(np.int64)), torch.from_numpy(ts % page)
            for pool in (kp, vp):
                for ch in range(k):
                    rows = rng.standard_normal((len(ts), Hkv, d), dtype=np.float32)
                    pool[ch].transpose(1, 2)[at[0], at[1]] = torch.from_numpy(rows).to(tdt)
        self.kp, self.vp, self.T = kp, vp, T
        self.kd, self.vd = kp.double().numpy(), vp.double().numpy()

    def rows(self, pool, c, b, h, ts):
        ts = np.asarray(ts, dtype=np.int64)
        return pool[c, self.table[b, ts // self.P], h, ts % self.P]

    def queries(self, *lead, scale=1.0):
        q = torch.from_numpy(self.rng.standard_normal((*lead, self.Hq, self.d)) * scale).to(self.tdt)
        return q

    def session(self, table=None):
        k = self.k
        cfg = W.make_config(k, k, 64, self.Hq, self.Hkv, self.d, 1, self.P, self.dtype, list(range(k)))
        s = DecodeSession(cfg, self.B, self.num_pages, self.max_pages)
        s.k_pool.copy_(self.kp)
        s.v_pool.copy_(self.vp)
        return s

    def dev(self):
        return (torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lens).cuda())

    # ---------------------------------------------------------- references
    def attend(self, c, b, hq, q, ts):
        """(out [d], weights [len(ts)], bound) of one query row over slots ts;
        bound: how far fp32 arithmetic may move a score, in natural units."""
        h = hq // self.G
        if len(ts) == 0:
            return np.zeros(self.d), np.zeros(0), 0.0, 0.0
        K, V = self.rows(self.kd, c, b, h, ts), self.rows(self.vd, c, b, h, ts)
        s = K @ q / np.sqrt(self.d)
        e = np.exp(s - s.max())
        p = e / e.sum()
        # d products and their sum, the scale and the exponent's argument each
        # round once to 24 bits
        ds = (self.d + 8) * 2.0 ** -24 * float((np.abs(K) @ np.abs(q)).max()) / np.sqrt(self.d)
        return p @ V, p, ds, float(np.abs(V).max())

    def out_tol(self, ds, vmax):
        """Largest error of one output element: weights off by a factor
        e^(2 ds) and a few roundings; bf16 also rounds every weight entering
        the product and the result (2^-9 each, relative)."""
        t = (2 * ds + 64 * 2.0 ** -24) * vmax
        return t + (2 * 2.0 ** -9 * vmax if self.dtype == "bf16" else 0.0)


def check_rows(cache, got, want, ds, vmax):
    got = np.asarray(got, np.float64)
    assert np.isfinite(got).all()
    err = np.abs(got - want).max()
    tol = cache.out_tol(ds, vmax)
    assert err <= tol, (err, tol)


def to_f64(t):
    return t.detach().cpu().double().numpy()
