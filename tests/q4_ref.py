"""The 4-bit paged cache and the rotation before it in 64 bits, from their definitions (include/kvd.h).  numpy only."""
from __future__ import annotations

import math

import numpy as np

D, TILE, TILE_BYTES = 128, 16, 2176
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EXP_MIN, EXP_MAX = -96, 125


def number(code, exp):
    """What codes stand for, exp of the same shape."""
    c = np.asarray(code, dtype=np.int64)
    return np.where(c & 8, -1.0, 1.0) * MAGNITUDES[c & 7] * np.exp2(np.asarray(exp, dtype=np.float64))


def exponent(amax):
    """The least e >= -96 with amax <= 7 * 2^e, at most 125."""
    e = EXP_MIN
    while e < EXP_MAX and amax > 7.0 * 2.0 ** e:
        e += 1
    return e


def quantise(x):
    """Codes [..., D] and exponents [..., D / 32] of elements."""
    x = np.array(x, dtype=np.float64)
    x[np.isnan(x)] = 0.0
    y = x.reshape(x.shape[:-1] + (4, 32))
    amax = np.where(np.isinf(y), 0.0, np.abs(y)).max(-1)
    exps = np.array([exponent(a) for a in amax.flatten()], dtype=np.int64).reshape(amax.shape)
    with np.errstate(over="ignore"):
        z = np.minimum(np.abs(y) * np.exp2(-exps.astype(np.float64))[..., None], 6.0)
    off = np.abs(z[..., None] - MAGNITUDES)                  # distances from all codes: the nearest, of two the even one
    best = off.min(-1, keepdims=True)
    order = np.where(off == best, np.arange(8) % 2, 9)
    code = order.argmin(-1)
    return (code | np.where(np.signbit(y), 8, 0)).reshape(x.shape), exps


def places(P):
    """Of every token and element of a page of P tokens: the keys' code and the values' (twice the byte, and 1 for the upper bits), and
    the bytes of their scales [P][4]."""
    t, d = np.arange(P)[:, None], np.arange(D)[None, :]
    tile, i = t // TILE * TILE_BYTES, t % TILE
    key = 2 * (tile + i * 64 + d // 2) + d % 2
    val = 2 * (tile + 1024 + d // 32 * 256 + d % 16 * 16 + d // 16 % 2 * 8 + i // 2) + i % 2
    g = np.arange(4)[None, :]
    return key, val, tile + 2048 + g * 16 + i % 4 * 4 + i // 4, tile + 2112 + g * 16 + i


class Cache:
    """codes [NB][H][2][P][D] and exps [NB][H][2][P][4] of keys and values."""

    def __init__(self, NB, H, P):
        self.NB, self.H, self.P = NB, H, P
        self.codes = np.zeros((NB, H, 2, P, D), dtype=np.int64)
        self.exps = np.full((NB, H, 2, P, 4), -127, dtype=np.int64)

    @classmethod
    def of_bytes(cls, pages, P):
        NB, H = pages.shape[:2]
        c = cls(NB, H, P)
        raw = np.asarray(pages).reshape(NB, H, -1).astype(np.int64)
        for which, (code, scale) in enumerate(zip(places(P)[:2], places(P)[2:])):
            c.codes[:, :, which] = raw[..., code // 2] >> (code % 2 * 4) & 15
            c.exps[:, :, which] = raw[..., scale] - 127
        return c

    def bytes(self):
        raw = np.zeros((self.NB, self.H, self.P // TILE * TILE_BYTES), dtype=np.int64)
        for which, (code, scale) in enumerate(zip(places(self.P)[:2], places(self.P)[2:])):
            for high in (0, 1):
                at = code % 2 == high
                raw[..., code[at] // 2] |= self.codes[:, :, which][..., at] << (4 * high)
            raw[..., scale] = self.exps[:, :, which] + 127
        return raw.reshape(self.NB, self.H, self.P // TILE, TILE_BYTES).astype(np.uint8)

    def append(self, runs, k, v):
        T = len(k)
        for block, row, off, n in runs:
            if not (0 <= block < self.NB and off >= 0 and n >= 1 and off + n <= self.P and row >= 0 and row + n <= T):
                continue
            if off == 0:
                self.codes[block, :, :, n:] = 0
                self.exps[block, :, :, n:] = EXP_MIN
            for which, x in enumerate((k, v)):
                code, e = quantise(x[row:row + n].transpose(1, 0, 2))
                self.codes[block, :, which, off:off + n], self.exps[block, :, which, off:off + n] = code, e

    def values(self, blocks, h, which):
        """[tokens][D] of the pages of `blocks`; those of blocks that are none are NaN."""
        blocks = np.asarray(blocks)
        good = (blocks >= 0) & (blocks < self.NB)
        b = np.where(good, blocks, 0)
        x = number(self.codes[b, h, which], np.repeat(self.exps[b, h, which], 32, -1))
        x[~good] = np.nan
        return x.reshape(-1, D)


class Row:
    """Attention of one row's query heads x [G][D] of a KV head, and what its error is measured by."""

    def __init__(self, ref, blocks, x, h, pos, lo, hi, scale, cap=0.0, slopes=None):
        k, v = ref.values(blocks, h, 0), ref.values(blocks, h, 1)
        t = np.arange(len(k))
        seen = (t >= lo) & (t <= hi) & ~np.isnan(k[:, 0])
        k, v, t = k[seen], v[seen], t[seen]
        self.empty = not len(t)
        if self.empty:
            return
        z = x @ k.T * scale
        if cap:
            z = cap * np.tanh(z / cap)
        self.capped = np.abs(z).max(-1)
        if slopes is not None:
            z = z - slopes[:, None] * np.abs(pos - t)[None, :]
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(-1, keepdims=True)
        p /= total
        self.n = len(t)
        self.out, self.lse = p @ v, (np.log(total) + top)[:, 0]
        self.mass = p @ np.abs(v)
        self.products = np.abs(x) @ np.abs(k).max(0) * scale               # no sum of |q k| is larger
        self.largest = np.abs(z).max(-1)
        self.bias = 0.0 if slopes is None else slopes * np.abs(pos - t).max()


def rotate(x, pos, inv_freq, *, interleaved=False, axis_pairs=None, weight=None, eps=1e-6):
    """Heads x [T][heads][D] at positions [axes][T], and a bound of what an element is made of."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    n = len(inv_freq)
    axis = np.repeat(np.arange(len(pos)), axis_pairs if axis_pairs is not None else [n])
    two_pi = 2 * math.pi
    turn = np.array([[math.fmod(float(pos[a][t]) * float(f), two_pi) for a, f in zip(axis, inv_freq)] for t in range(len(x))])
    i = np.arange(n)
    one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    y, size = x.copy(), np.abs(x)
    if n:
        c, s = np.cos(turn)[:, None], np.sin(turn)[:, None]
        a, b = x[..., one], x[..., two]
        y[..., one], y[..., two] = a * c - b * s, a * s + b * c
        size[..., one] = size[..., two] = np.abs(a) + np.abs(b)
    return y, size
