"""Plain implementations in 64 bits (numpy, loops) of the cache, attention and log-probability operators, and helpers
that build paged caches for their GPU tests. Nothing here imports the library."""
from __future__ import annotations

import numpy as np

BLOCK = 32


def bf16_round(x):
    """float32 array rounded to the nearest bf16 (ties to even), as float32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16
    return r.astype(np.uint32).view(np.float32).reshape(np.shape(x))


def bf16_bits(x):
    """uint16 patterns of values that are exact in bf16."""
    return (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16).reshape(np.shape(x))


def bits_to_f64(bits):
    return (np.asarray(bits, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)


def _e4m3_table():
    t = np.zeros(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        t[c] = np.nan if (c & 127) == 127 else (-v if s else v)
    return t


E4M3 = _e4m3_table()
_POS = E4M3[:127]                               # ascending magnitudes, code = index


def e4m3_codes(x):
    """Nearest E4M3 codes (ties to the even code) of values of magnitude at most 448; the sign of zero is kept, NaN is 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    nan = np.isnan(x)
    x = np.where(nan, 0.0, x)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.clip(hi - 1, 0, 126)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(_POS[hi] == a, hi, code)
    return np.where(nan, 0x7F, code + 128 * np.signbit(x)).astype(np.uint8)


def scale_of(amax):
    """Smallest power of two s >= 2^-64 with amax <= 448 s."""
    s = 2.0 ** -64
    while s * 448.0 < amax:
        s *= 2.0
    return s


def rotate(x, pos, cos, sin, rot, style):
    """One head of one token, every product and sum rounded to float32, as the operator defines it."""
    y = x.astype(np.float32).copy()
    f = np.float32
    for i in range(rot // 2):
        a, b = (i, i + rot // 2) if style == "half" else (2 * i, 2 * i + 1)
        c, s = f(cos[pos, i]), f(sin[pos, i])
        u, v = f(x[a]), f(x[b])
        with np.errstate(invalid="ignore", over="ignore"):
            y[a] = f(f(u * c) - f(v * s))
            y[b] = f(f(v * c) + f(u * s))
    return y


def rotate64(x, pos, cos, sin, rot, style):
    y = x.astype(np.float64).copy()
    for i in range(rot // 2):
        a, b = (i, i + rot // 2) if style == "half" else (2 * i, 2 * i + 1)
        z = complex(x[a], x[b]) * complex(cos[pos, i], sin[pos, i])
        y[a], y[b] = z.real, z.imag
    return y


def attend(q, k, v, scale, first, last):
    """One row over keys [first, last): (out, lse, sum p|v|, largest sum |q||k| scale) in 64 bits."""
    d = q.shape[0]
    if last <= first:
        return np.zeros(d), -np.inf, np.zeros(d), 0.0
    k, v = k[first:last], v[first:last]
    x = (k @ q) * scale
    m = x.max()
    e = np.exp(x - m)
    p = e / e.sum()
    return p @ v, m + np.log(e.sum()), p @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * scale)


def seen(length, n, r, causal, window):
    """The range of keys that query row r of n sees in a context of `length` tokens."""
    if not causal:
        return 0, length
    p = length - n + r
    return (max(0, p - window + 1) if window else 0), max(0, p + 1)


def logprobs(x, target, n_top):
    """One row of logits in 64 bits: (lp of the target, entropy, ids, lps, sum p |x - m|)."""
    x = np.asarray(x, dtype=np.float64)
    order = sorted(range(x.size), key=lambda i: (-x[i], i))[:n_top]
    m = x.max()
    if m == -np.inf:
        return (0.0 if not 0 <= target < x.size else -np.inf), 0.0, order, [-np.inf] * n_top, 0.0
    e = np.exp(x - m)
    lse = m + np.log(e.sum())
    p = e / e.sum()
    live = p > 0
    h = -np.sum(p[live] * (x[live] - lse))
    lp = x[target] - lse if 0 <= target < x.size else 0.0
    return lp, h, order, [x[i] - lse for i in order], float(np.sum(p[live] * np.abs(x[live] - m)))


class Paged:
    """A paged cache in numpy: pools of one layer with every slot holding NaN until it is written, scales, block table."""

    def __init__(self, kv, d, page, widths, e4m3, layout="HND", pad=0, spare=2, seed=0, table_tokens=0):
        rng = np.random.default_rng([26, seed])
        self.kv, self.d, self.page, self.e4m3, self.layout = kv, d, page, e4m3, layout
        self.n_pages = int(sum(widths)) + spare
        row = d + pad                               # padding between tokens' rows
        if layout == "HND":
            self.stride_token, self.stride_head, self.page_stride = row, page * row, kv * page * row
        else:
            self.stride_token, self.stride_head, self.page_stride = kv * row, row, page * kv * row
        size = self.n_pages * self.page_stride
        dt = np.uint8 if e4m3 else np.uint16
        self.k = np.full(size, 0x7F if e4m3 else 0x7FC0, dtype=dt)
        self.v = self.k.copy()
        self.ks = np.full((self.n_pages, kv, page // BLOCK), np.nan, dtype=np.float32)
        self.vs = self.ks.copy()
        entries = max(max(widths, default=1), 1, -(-table_tokens // page))
        self.table = np.full((len(widths), entries), -1, dtype=np.int32)
        perm = rng.permutation(self.n_pages)
        at = 0
        for b, w in enumerate(widths):
            self.table[b, :w] = perm[at:at + w]
            at += w

    def at(self, b, kv, j):
        """Element offset of a token's row."""
        page = int(self.table[b, j // self.page])
        return page * self.page_stride + kv * self.stride_head + (j % self.page) * self.stride_token

    def scale_at(self, b, kv, j):
        return int(self.table[b, j // self.page]), kv, j % self.page // BLOCK

    def fill(self, b, k, v):
        """Tokens [L][kv][d] of request b from the start, quantised where the cache is; returns the values held."""
        held = []
        for pool, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            y = np.zeros_like(x, dtype=np.float64)
            for j0 in range(0, x.shape[0], BLOCK):
                for h in range(self.kv):
                    part = x[j0:j0 + BLOCK, h].astype(np.float64)
                    s = scale_of(np.abs(part).max()) if self.e4m3 else 1.0
                    if self.e4m3:
                        scales[self.scale_at(b, h, j0)] = s
                    for i, row in enumerate(part):
                        o = self.at(b, h, j0 + i)
                        if self.e4m3:
                            pool[o:o + self.d] = e4m3_codes(row / s)
                            y[j0 + i, h] = E4M3[pool[o:o + self.d]] * s
                        else:
                            pool[o:o + self.d] = bf16_bits(bf16_round(row))
                            y[j0 + i, h] = bits_to_f64(pool[o:o + self.d])
            held.append(y)
        return held
