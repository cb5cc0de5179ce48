"""Builds steps of the 4-bit paged cache on the GPU and compares them with their 64-bit definition for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2605_18071_amd import kvd as K
from tests import q4_ref as R
from tests.q8_rig import DEV, D, i32, torch_type


class Step:
    """Sequences of `lens` tokens that get `news` more, in a pool of random codes and scales."""

    def __init__(self, lens, news, *, P=16, H=2, G=4, dtype="bf16", seed=0, spare=0, max_pages=None, blocks=None, scale=0.0, exps=(-3, 1)):
        self.lens, self.news, self.P, self.H, self.G, self.dtype = list(lens), list(news), P, H, G, dtype
        B = len(lens)
        ends = [a + n for a, n in zip(lens, news)]
        need = [-(-e // P) for e in ends]
        NP = max_pages or max(max(need), 1)
        NB = blocks or sum(need) + 3
        rng = np.random.default_rng(seed)
        self.table = np.full((B, NP), -1, dtype=np.int64)
        order = rng.permutation(NB)
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        T = max(1, sum(news)) + spare
        self.T, self.real, self.NB, self.scale = T, sum(news), NB, scale
        self.seq = [b for b, n in enumerate(news) for _ in range(n)]
        self.pos = [a + i for a, n in zip(lens, news) for i in range(n)]
        start = np.concatenate([[0], np.cumsum(news)])
        runs = []
        for r, (b, p) in enumerate(zip(self.seq, self.pos)):
            if p == lens[b] or p % P == 0:
                runs.append([int(self.table[b, p // P]), r, p % P, 0])
            runs[-1][3] += 1
        self.runs = runs + [[-1, 0, 0, 0]] * (1 + spare)
        pad = [-1] * (T - len(self.seq))
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)
        pages = torch.empty((NB, H, P // 16, 2176), dtype=torch.uint8, device=DEV)
        pages.copy_(torch.randint(0, 256, pages.shape, generator=self.gen, device=DEV))
        pages[..., 2048:] = torch.randint(127 + exps[0], 127 + exps[1], pages[..., 2048:].shape, generator=self.gen, device=DEV).to(torch.uint8)
        self.cache = K.Q4Cache(n_blocks=NB, n_q_heads=H * G, n_kv_heads=H, page_size=P, kv_dtype=torch_type(dtype), softmax_scale=scale, pages=pages)
        self.rows = K.Q8Rows(i32(self.table), page_size=P, n_blocks=NB, n_rows=T, max_runs=len(self.runs), kv_len=i32(ends),
                             row_start=i32(start), row_seq=i32(self.seq + pad), row_pos=i32(self.pos + pad), runs=i32(self.runs))

    def ref(self):
        return R.Cache.of_bytes(self.cache.pages.cpu().numpy(), self.P)

    def randn(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.gen, device=DEV) * scale).to(torch_type(self.dtype))

    def query(self, scale=1.0):
        return self.randn(self.T, self.H * self.G, D, scale=scale)

    def attend(self, q, *, lse=True, ws=None, stream=None, **kw):
        out = torch.full((self.T, self.H * self.G, D), 7.0, dtype=q.dtype, device=DEV)
        ls = torch.full((self.T, self.H * self.G), 7.0, dtype=torch.float32, device=DEV) if lse else None
        kw = {n: v if v is None or isinstance(v, (int, float)) else torch.as_tensor(v, device=DEV) for n, v in kw.items()}
        self.cache.attend(self.rows, q, out, self.cache.workspace(self.rows) if ws is None else ws, lse=ls, stream=stream, **kw)
        return out, ls

    def check(self, q, out, lse, *, rows=None, table=None, softcap=0.0, window=0, slopes=None, row_from=None, prefix_len=None, weights=None):
        """Rows against the 64-bit definition.  With A = sum p |v| / sum p, an output is off by at most
           half a step of its type                                                                     h |o|
         + the weights' rounding to bf16, half a step of 8 bits: 2^-8 (f16: the rest's, 2^-16)         r A
         + twice the logits' error and the sums' and joins' 2^-17                                      A
         + what fp32 cannot hold: weights times scales are kept with the row's largest weight at 2^-36, and what is below fp32's least
           normal 2^-126 may be lost: 2^(36 - 126) of a code of up to 6 for each token                            n 2^-87
         + f16: below its normal numbers                                                               2^-25.
        `weights`: r, where that has to be less.
        Logits: products of 128 elements and their sums in fp32 (2^-17 sum |q k| scale), a cap's exponent and reciprocal (2^-20 of the
        cap; above 64 of the logit), a bias's rounding (2^-22), the exponent's argument (2^-23 of it) and 2^-20."""
        ref, table = self.ref(), self.table if table is None else table
        h = torch.finfo(torch_type(self.dtype)).eps / 2
        r = weights or (2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -16)
        scale = self.scale or 1.0 / math.sqrt(D)
        qd, od, ld = q.double().cpu().numpy(), out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
        sl = None if slopes is None else np.asarray(slopes, dtype=np.float64)
        for row in (range(self.real) if rows is None else rows):
            b, pos = self.seq[row], self.pos[row]
            end = self.lens[b] + self.news[b]
            lo = max(0, pos - window + 1) if window else 0
            if row_from is not None:
                lo = max(lo, int(row_from[row]))
            hi = max(pos, min(int(prefix_len[b]), end) - 1) if prefix_len is not None else pos
            for hd in range(self.H):
                heads = slice(hd * self.G, (hd + 1) * self.G)
                x = R.Row(ref, table[b], qd[row, heads], hd, pos, lo, hi, scale, softcap, None if sl is None else sl[heads])
                got = od[row, heads]
                if x.empty:
                    assert (got == 0).all() and (ld is None or (ld[row, heads] == -np.inf).all()), (row, hd)
                    continue
                dx = 2.0 ** -17 * x.products + 2.0 ** -20 * (1 + (softcap if softcap <= 64 else x.capped)) + 2.0 ** -22 * x.bias + 2.0 ** -23 * x.largest
                tol = h * np.abs(x.out) + (r + 2 * dx[:, None] + 2.0 ** -17) * x.mass + x.n * 2.0 ** -87
                if self.dtype == "f16":
                    tol = tol + 2.0 ** -25
                bad = ~(np.abs(got - x.out) <= tol)
                assert not bad.any(), f"row {row} head {hd}: {np.abs(got - x.out)[bad].max()} over {tol[bad].min()}, {bad.sum()} of {bad.size}"
                if ld is not None:
                    assert (np.abs(ld[row, heads] - x.lse) <= dx + 2.0 ** -20 * (1 + np.abs(x.lse))).all(), (row, hd)
        # rows without a sequence stay as they were
        assert (od[self.real:] == 7.0).all() and (ld is None or (ld[self.real:] == 7.0).all())
