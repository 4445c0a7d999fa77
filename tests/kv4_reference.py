"""The 4-bit key/value cache from its definition, in NumPy: codes and layouts bit for bit, attention in 64 bits."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([VALUES, -VALUES])


def block_of(d):
    return min(128, d & -d)


def walsh(x, block):
    """Sums and differences of neighbours, of pairs apart by 2, by 4 ..; without the factor.  In x's type."""
    step, shape = 1, x.shape
    while step < block:
        p = x.reshape(shape[:-1] + (shape[-1] // (2 * step), 2, step))
        x = np.stack([p[..., 0, :] + p[..., 1, :], p[..., 0, :] - p[..., 1, :]], -2).reshape(shape)
        step *= 2
    return x


def factor(block):
    """block^-1/2 in fp32: a power of two, times the root of a half rounded to fp32."""
    k = block.bit_length() - 1
    return np.float32((np.float32(np.sqrt(0.5)) if k & 1 else np.float32(1)) * np.float32(2.0 ** -(k // 2)))


BORDERS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])


def codes_of(t):
    """E2M1 to nearest, ties to even."""
    a = np.abs(t)[..., None]
    up = np.where(np.arange(7) % 2 == 0, a > BORDERS, a >= BORDERS)     # at a border the even code wins
    return (up.sum(-1) + 8 * np.signbit(t)).astype(np.uint8)


def exact_codes(sums, least=None):
    """The codes that the definition gives for heads of sums [.., d] in 64 bits, in units of any size: 6 |sum| / max |sum| against the borders, by
    products that are exact for sums of up to 47 bits.  least: the smallest that the largest counts as."""
    a, top = np.abs(sums), np.abs(sums).max(-1, keepdims=True)
    top = np.where(top == 0, 1, top) if least is None else np.maximum(np.where(top == 0, 1, top), least)
    up = np.where(np.arange(7) % 2 == 0, 6 * a[..., None] > BORDERS * top[..., None], 6 * a[..., None] >= BORDERS * top[..., None])
    return (up.sum(-1) + 8 * (sums < 0)).astype(np.uint8)


def encode(z):
    """(codes, scales) of heads as transformed() gives them: codes from the sums in 64 bits, scales by 32-bit steps."""
    sums, steps, f = z
    with np.errstate(all="ignore"):
        top = np.abs(steps).max(-1)
        scale = np.where(top == 0, np.float32(1), np.maximum(top / np.float32(6), np.float32(2.0 ** -126))).astype(np.float32)
        good = np.isfinite(top)
        codes = np.where(good[..., None], exact_codes(np.where(good[..., None], sums, 0), 6 * 2.0 ** -126 / f), 0)
    return codes.astype(np.uint8), np.where(good, scale, np.float32(np.nan))


def transformed(x, block):
    """Of heads x: the sums in 64 bits, the transform by 32-bit steps, the factor between them."""
    with np.errstate(all="ignore"):
        return walsh(x.astype(np.float64), block), walsh(x.astype(np.float32), block) * factor(block), block ** -0.5


class Cache:
    """codes [pages, kv_heads, page_size, d] and scales [pages, kv_heads, page_size], of keys and of values"""

    def __init__(self, pages, heads, page, d, rng=None, scale=1.0):
        self.pages, self.heads, self.page, self.d = pages, heads, page, d
        shape = (pages, heads, page)
        if rng is None:
            self.k, self.v = np.zeros(shape + (d,), np.uint8), np.zeros(shape + (d,), np.uint8)
            self.ks, self.vs = np.zeros(shape, np.float32), np.zeros(shape, np.float32)
        else:
            self.k, self.v = (rng.integers(0, 16, shape + (d,), dtype=np.uint8) for _ in "kv")
            self.ks, self.vs = (np.float32(scale) * np.exp(rng.normal(-1, 0.5, shape)).astype(np.float32) for _ in "kv")

    def packed(self):
        """As the library keeps it."""
        pitch = -(-self.d // 32) * 32
        wide = lambda x: np.pad(x, [(0, 0)] * 3 + [(0, pitch - self.d)])
        k, v = wide(self.k), wide(self.v)
        k = k[..., 0::2] | k[..., 1::2] << 4
        v = v.reshape(self.pages, self.heads, self.page // 8, 8, pitch).swapaxes(3, 4)
        return k, np.ascontiguousarray(v[..., 0::2] | v[..., 1::2] << 4), self.ks, self.vs

    def unpack(self, k, v, ks, vs):
        k, v = k[..., :self.d // 2], v[..., :self.d, :]
        self.k = np.stack([k & 15, k >> 4], -1).reshape(self.ks.shape + (self.d,))
        self.v = np.stack([v & 15, v >> 4], -1).reshape(self.pages, self.heads, self.page // 8, self.d, 8).swapaxes(3, 4).reshape(self.k.shape)
        self.ks, self.vs = ks, vs
        return self

    def rows(self, table, length):
        """(k, v) [length, heads, d]: numbers in the transformed basis, 64 bits; NaN where there is no page."""
        place = np.arange(length)
        column = place // self.page
        page = np.where(column < len(table), table[np.minimum(column, len(table) - 1)], -1)
        good = (page >= 0) & (page < self.pages)
        at = (np.where(good, page, 0), slice(None), place % self.page)
        out = []
        for codes, scales in ((self.k, self.ks), (self.v, self.vs)):
            x = VALUES[codes[at]] * scales[at].astype(np.float64)[..., None]
            out.append(np.where(good[:, None, None], x, np.nan))
        return out


def attention(q, cache, table, lengths, begins, scale, window, sinks, block, wide, least=2.0 ** -25):
    """(out, bound) [t, heads, d] in 64 bits: the definition, and how far a kernel may be from it before its result is rounded.

    Roundings counted (u = 2^-11, half a step of a half; two halves 2^-22): of H q, of the weights times the scales of v, where the largest weight is
    1 and the power of two next to the largest scale is taken out; small products are off by `least` of that scale.  fp32: sums of d and of n
    terms in any order, with 2^-23 a step; the
    exponential's argument by 2^-23 of itself.  An error e of every score changes a result by at most (exp(2 e) - 1) of sum p |v|."""
    t, heads, d = q.shape
    group, u = heads // cache.heads, 2.0 ** -22 if wide else 2.0 ** -11
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    hq = walsh(q.astype(np.float64), block) / np.sqrt(block)
    size = np.abs(walsh(np.eye(d), block)) / np.sqrt(block)
    most = 6 * np.nanmax(cache.vs)
    for b, length in enumerate(lengths):
        rows = np.arange(begins[b], begins[b + 1])
        n, length = len(rows), max(0, int(length))
        if length > len(table[b]) * cache.page:
            out[rows] = np.nan
            continue
        k, v = cache.rows(table[b], length)
        j = np.arange(length)
        for i, row in enumerate(rows):
            pos = length - n + i
            seen = j <= pos
            if window:
                seen &= (j > pos - window) | (j < sinks)
            if not seen.any():
                continue
            for h in range(heads):
                kk, vv = k[seen, h // group], v[seen, h // group]
                s = scale * (kk @ hq[row, h])
                if not np.isfinite(s).all() or not np.isfinite(vv).all():
                    out[row, h] = np.nan
                    continue
                top = s.max()
                p = np.exp(s - top)
                p /= p.sum()
                e = abs(scale) * (np.abs(kk) @ np.abs(hq[row, h])) * (u + 2.0 ** -22 + (d + 16) * 2.0 ** -23) + (np.abs(s - top) + 16) * 2.0 ** -22
                grow = np.expm1(2 * e.max()) + u + (len(s) + 64) * 2.0 ** -23
                off = grow * (p @ np.abs(vv)) + len(s) * least * most * p.max()
                out[row, h] = walsh(p @ vv, block) / np.sqrt(block)
                bound[row, h] = size @ off + 2.0 ** -20 * (size @ (p @ np.abs(vv)))
    return out, bound
