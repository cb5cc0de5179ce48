"""Plain 64-bit definition of the 8-bit paged cache (CPU, numpy): page tables, appending, selection, attention.
Loops over sequences, pages and heads; nothing in it is shared with the library."""
from __future__ import annotations

import math

import numpy as np

D = 128
EXP_MIN = -96

# the 256 values of e4m3: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are no numbers
_c = np.arange(256)
_ex, _man = (_c >> 3) & 15, _c & 7
VALUES = np.where(_ex == 0, _man * 2.0 ** -9, (8 + _man) * 2.0 ** (_ex - 10.0)) * np.where(_c >> 7, -1.0, 1.0)
VALUES[[0x7F, 0xFF]] = np.nan
_POS = VALUES[:0x7F]                                   # ascending


def encode(x):
    """Nearest code of each |x| <= 448, ties to the even code."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POS, a, side="left"), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def exp_for(x):
    """Least e >= EXP_MIN with every finite |x| <= 448 * 2^e."""
    a = np.abs(x[np.isfinite(x)])
    top = float(a.max()) if a.size else 0.0
    if top == 0.0:
        return EXP_MIN
    e = math.ceil(math.log2(top / 448.0)) - 2
    while top > math.ldexp(448.0, e):
        e += 1
    return max(e, EXP_MIN)


def quantise(x, e):
    y = np.where(np.isnan(x), 0.0, x) * math.ldexp(1.0, -e)
    return encode(np.clip(y, -448.0, 448.0))


def tile_places(P):
    """(key, value) byte of token t, element d inside a page, [P][D]."""
    t, d = np.arange(P)[:, None], np.arange(D)[None, :]
    i, tile = t % 16, t // 16 * 4096
    key = tile + d // 64 * 1024 + (d // 8 % 4 * 16 + i) * 16 + d // 32 % 2 * 8 + d % 8
    val = tile + 2048 + d // 64 * 1024 + (i // 4 * 16 + d % 16) * 16 + d // 16 % 4 * 4 + i % 4
    return key, val


class Cache:
    def __init__(self, NB, H, P):
        self.NB, self.H, self.P = NB, H, P
        self.codes = np.zeros((NB, H, 2, P, D), dtype=np.uint8)
        self.exps = np.zeros((NB, H, 2), dtype=np.int64)
        self.means = np.zeros((NB, H, D), dtype=np.int8)
        self.mean_scales = np.zeros((NB, H), dtype=np.float32)

    def append(self, runs, k, v):
        """runs [n][4]; k, v [T][H][D] in 64 bits."""
        for block, row, off, n in runs:
            if not (0 <= block < self.NB and off >= 0 and n >= 1 and off + n <= self.P and row >= 0 and row + n <= len(k)):
                continue
            for h in range(self.H):
                for w, x in enumerate((k, v)):
                    new = x[row:row + n, h]
                    e, was = exp_for(new), int(self.exps[block, h, w])
                    c = self.codes[block, h, w]
                    if off == 0:
                        c[:] = 0
                    elif e > was:
                        c[:off] = encode(VALUES[c[:off]] * math.ldexp(1.0, was - e))
                    else:
                        e = was
                    c[off:off + n] = quantise(new, e)
                    self.exps[block, h, w] = e
                S = (VALUES[self.codes[block, h, 0, :off + n]] * 512.0).sum(0)
                sh = 0
                while np.abs(S).max() > 127 * 2 ** sh:
                    sh += 1
                self.means[block, h] = np.round(S / 2 ** sh).astype(np.int8)
                self.mean_scales[block, h] = np.float32(math.ldexp(1.0, sh - 9 + int(self.exps[block, h, 0])) / (off + n))

    def bytes(self):
        """[NB][H][P/16][2][2048] as the library lays them out."""
        key, val = tile_places(self.P)
        out = np.zeros((self.NB, self.H, self.P * 2 * D), dtype=np.uint8)
        out[..., key] = self.codes[:, :, 0]
        out[..., val] = self.codes[:, :, 1]
        return out.reshape(self.NB, self.H, self.P // 16, 2, 2048)

    def kv(self, blocks, h):
        """Keys and values [tokens][D] of one head's pages; bad blocks give zeros."""
        got = []
        for w in range(2):
            x = [VALUES[self.codes[b, h, w]] * math.ldexp(1.0, int(self.exps[b, h, w])) if 0 <= b < self.NB
                 else np.zeros((self.P, D)) for b in blocks]
            got.append(np.concatenate(x) if x else np.zeros((0, D)))
        return got


def map_step(seq_len, n_new, table, free, free_count, P, T, R):
    """What kvd_q8_map writes; table is changed in place."""
    B, NP = table.shape
    have = min(max(int(free_count), 0), len(free))
    why = 0
    ok = [l >= 0 and n >= 0 and l + n <= NP * P for l, n in zip(seq_len, n_new)]
    why |= 0 if all(ok) else 8
    if any(o and n > T for o, n in zip(ok, n_new)) or sum(n for o, n in zip(ok, n_new) if o) > T:
        why |= 2
    row_start, row_seq, row_pos, runs, taken = [0], [], [], [], 0
    new_table = table.copy()
    for b, (l, n) in enumerate(zip(seq_len, n_new)):
        if not ok[b] or n > T:
            n = 0
            l = 0
        for p in range(-(-l // P), -(-(l + n) // P)):
            new_table[b, p] = free[have - 1 - taken] if taken < have else -7
            taken += 1
        r0 = len(row_seq)
        for i in range(n):
            row_seq.append(b)
            row_pos.append(l + i)
            if i == 0 or (l + i) % P == 0:
                runs.append([int(new_table[b, (l + i) // P]), r0 + i, (l + i) % P, 0])
            runs[-1][3] += 1
        row_start.append(len(row_seq))
    if taken > have:
        why |= 1
    if len(runs) > R:
        why |= 4
    if why:
        return dict(kv_len=list(seq_len), row_start=[0] * (B + 1), row_seq=[-1] * T, row_pos=[-1] * T,
                    runs=[[-1, 0, 0, 0]] * R, counts=[0, 0, 0, have, why])
    table[:] = new_table
    n = len(row_seq)
    return dict(kv_len=[l + n for l, n in zip(seq_len, n_new)], row_start=row_start, row_seq=row_seq + [-1] * (T - n),
                row_pos=row_pos + [-1] * (T - n), runs=runs + [[-1, 0, 0, 0]] * (R - len(runs)),
                counts=[n, len(runs), taken, have - taken, 0])


def select_row(cache, table_row, q, h, pos, k, sink, recent, NB):
    """Pages of one row and head: q [G][D] in 64 bits, exact sums."""
    P = cache.P
    n = pos // P + 1
    s = q.sum(0)
    m = np.abs(s).max()
    with np.errstate(all="ignore"):
        y = s * (np.float64(127.0) / np.float64(m))
    qi = np.where(np.isfinite(y), np.round(np.where(np.isfinite(y), y, 0.0)), 0.0)
    score = np.full(n, -np.inf)
    for p in range(n):
        b = table_row[p]
        if 0 <= b < NB:
            score[p] = np.float32(np.float32(qi @ cache.means[b, h].astype(np.float64)) * cache.mean_scales[b, h])
    score[:sink] = np.inf
    if recent:
        score[max(0, n - recent):] = np.inf
    best = sorted(sorted(range(n), key=lambda p: (-score[p], p))[:k])
    return best + [-1] * (k - len(best))


def attend_row(cache, table_row, q, h, pos, scale, pages=None):
    """(out [G][D], lse [G]) of one row and head in 64 bits."""
    P = cache.P
    if pages is None:
        pages = range(pos // P + 1)
    pages = [p for p in pages if p >= 0]
    k, v = cache.kv([table_row[p] for p in pages], h)
    at = np.concatenate([np.arange(p * P, p * P + P) if 0 <= table_row[p] < cache.NB else np.full(P, 1 << 40) for p in pages]) \
        if pages else np.zeros(0)
    see = at <= pos
    if not see.any():
        return np.zeros((len(q), D)), np.full(len(q), -np.inf)
    x = q @ k[see].T * scale
    m = x.max(1, keepdims=True)
    p = np.exp(x - m)
    l = p.sum(1, keepdims=True)
    return (p @ v[see]) / l, (m + np.log(l))[:, 0]
