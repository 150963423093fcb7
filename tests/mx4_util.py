"""Microscaled 4-bit elements in 64 bits (numpy), and paged caches of them for the GPU tests. Nothing here imports the library."""
from __future__ import annotations

import numpy as np

import operator_util as ou

GROUP = 32
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([E2M1, -E2M1])


def nearest(z):
    """Codes 0 .. 7 of magnitudes of at most 6: the nearest, of two as near the even one."""
    d = np.abs(z[..., None] - E2M1)
    return np.argmin(d + np.where(np.arange(8) % 2, 1e-9, 0) * (d > 0), axis=-1).astype(np.uint8)


def quantise(x):
    """[..., n] -> codes [..., n] (one each) and scale bytes [..., n / 32], by the definition."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    bad = ~np.isfinite(y).all(axis=-1)
    y = np.where(bad[..., None], 0.0, y)
    m = np.abs(y).max(axis=-1)
    e = np.full(m.shape, -64)
    while (over := m > 6 * np.exp2(e.astype(np.float64))).any():
        e = e + over
    codes = nearest(np.abs(y) / np.exp2(e.astype(np.float64))[..., None]) + 8 * np.signbit(y).astype(np.uint8)
    codes = np.where(bad[..., None], 0, codes).astype(np.uint8)
    return codes.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(codes):
    """Two codes to a byte, the lower element in the lower bits."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(b):
    return np.stack([b & 15, b >> 4], axis=-1).reshape(*b.shape[:-1], 2 * b.shape[-1])


def values(codes, scales):
    """What codes (one each) and scale bytes stand for."""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return VALUES[codes] * np.repeat(s, GROUP, axis=-1)


class Paged4(ou.Paged):
    """A paged cache of 4-bit elements: slots that have not been written hold any codes, and scales that say NaN."""

    def __init__(self, kv, d, page, widths, layout="HND", pad=0, spare=2, seed=0, table_tokens=0):
        super().__init__(kv, d, page, widths, False, layout, pad, spare, seed, table_tokens)
        rng = np.random.default_rng([27, seed])
        size = self.n_pages * self.page_stride // 2
        self.k, self.v = (rng.integers(0, 256, size).astype(np.uint8) for _ in range(2))
        self.ks, self.vs = (np.full((self.n_pages, kv, page, d // GROUP), 255, dtype=np.uint8) for _ in range(2))

    def put(self, pool, scales, b, h, j, codes, scale):
        o = self.at(b, h, j) // 2
        pool[o:o + self.d // 2] = pack(codes)
        scales[int(self.table[b, j // self.page]), h, j % self.page] = scale

    def fill(self, b, k, v):
        """Tokens [L][kv][d] of request b from the start; returns the values held."""
        held = []
        for pool, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            codes, s = quantise(x)
            for j in range(x.shape[0]):
                for h in range(self.kv):
                    self.put(pool, scales, b, h, j, codes[j, h], s[j, h])
            held.append(values(codes, s))
        return held
