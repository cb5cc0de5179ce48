"""Builds steps of the 8-bit paged cache on the GPU and their 64-bit counterparts for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2605_18071_amd import kvd as K
from tests import q8_ref as R

DEV = "cuda"
D = 128


def torch_type(dtype):
    return torch.float16 if dtype == "f16" else torch.bfloat16


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def to_ref(cache: K.Q8Cache, P: int) -> R.Cache:
    """The library's buffers as the reference's: attention and selection are then compared on the same codes."""
    NB, H = cache.exps.shape[:2]
    ref = R.Cache(NB, H, P)
    key, val = R.tile_places(P)
    raw = cache.pages.cpu().numpy().reshape(NB, H, -1)
    ref.codes[:, :, 0], ref.codes[:, :, 1] = raw[..., key], raw[..., val]
    ref.exps = cache.exps.cpu().numpy().astype(np.int64)
    ref.means, ref.mean_scales = cache.means.cpu().numpy(), cache.mean_scales.cpu().numpy()
    return ref


class Step:
    """Sequences of `lens` tokens that get `news` more, in a pool of random codes and scales."""

    def __init__(self, lens, news, *, P=16, H=2, G=4, dtype="bf16", seed=0, spare=0, max_pages=None, blocks=None, **kw):
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
        self.T, self.real = T, sum(news)
        seq = [b for b, n in enumerate(news) for _ in range(n)]
        pos = [a + i for a, n in zip(lens, news) for i in range(n)]
        self.seq, self.pos = seq + [-1] * (T - len(seq)), pos + [-1] * (T - len(pos))
        start = np.concatenate([[0], np.cumsum(news)])
        runs = []
        for r, (b, p) in enumerate(zip(seq, pos)):
            if p == lens[b] or p % P == 0:
                runs.append([int(self.table[b, p // P]), r, p % P, 0])
            runs[-1][3] += 1
        self.runs = runs + [[-1, 0, 0, 0]] * (1 + spare)
        self.NB = NB
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.gen = g
        self.cache = K.Q8Cache(n_blocks=NB, n_q_heads=H * G, n_kv_heads=H, page_size=P, kv_dtype=torch_type(dtype), device=DEV, **kw)
        c = self.cache
        c.pages.copy_((torch.randn(c.pages.shape, generator=g, device=DEV) * 75).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
        c.exps.copy_(torch.randint(-8, -4, c.exps.shape, generator=g, device=DEV))
        c.means.copy_((torch.randn(c.means.shape, generator=g, device=DEV) * 40).round().clamp(-127, 127))
        c.mean_scales.copy_(torch.rand(c.mean_scales.shape, generator=g, device=DEV) * 0.01 + 0.001)
        self.rows = K.Q8Rows(i32(self.table), page_size=P, n_blocks=NB, n_rows=T, max_runs=len(self.runs), kv_len=i32(ends),
                             row_start=i32(start), row_seq=i32(self.seq), row_pos=i32(self.pos), runs=i32(self.runs))

    def randn(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.gen, device=DEV) * scale).to(torch_type(self.dtype))

    def query(self, scale=1.0):
        return self.randn(self.T, self.H * self.G, D, scale=scale)

    def attend(self, q, sel=None, lse=True, ws=None, stream=None):
        out = torch.full((self.T, self.H * self.G, D), 7.0, dtype=q.dtype, device=DEV)
        ls = torch.full((self.T, self.H * self.G), 7.0, dtype=torch.float32, device=DEV) if lse else None
        ws = self.cache.workspace(self.rows) if ws is None else ws
        self.cache.attend(self.rows, q, out, ws, lse=ls, sel_pages=sel, stream=stream)
        return out, ls

    def check_attention(self, q, out, lse, sel=None, rows=None, table=None):
        """Rows against the 64-bit definition.  With A = sum p |v| / sum p, an output is off by at most
           half a step of its type                                                    h |o|
         + what rounding P costs: 2^-16 with rows alone (P in two parts), else a half step   r A
         + twice the logits' error (128 products and their sums in fp32: 2^-17 sum |q k| scale; exponent, maximum: 2^-20)
           and the sums' and the joins' (2^-17)                                          A
         + f16: outputs below its normal numbers (2^-25) and weights below (2^-25 times the largest value, for each token)."""
        ref = to_ref(self.cache, self.P)
        table = self.table if table is None else table
        h = torch.finfo(torch_type(self.dtype)).eps / 2
        alone = sel is not None or self.T <= len(self.lens)
        r = 2.0 ** -16 if alone else h
        scale = 1.0 / math.sqrt(D)
        qd, od, ld = q.double().cpu().numpy(), out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
        sd = None if sel is None else sel.cpu().numpy()
        for row in (range(self.real) if rows is None else rows):
            b, pos = self.seq[row], self.pos[row]
            for hd in range(self.H):
                pages = None if sel is None else sd[row, hd]
                x = qd[row, hd * self.G:(hd + 1) * self.G]
                o, l = R.attend_row(ref, table[b], x, hd, pos, scale, pages)
                got = od[row, hd * self.G:(hd + 1) * self.G]
                if not np.isfinite(l).all():
                    assert (got == 0).all() and (ld is None or (ld[row, hd * self.G:(hd + 1) * self.G] == -np.inf).all()), (row, hd)
                    continue
                k, v = ref.kv(table[b][[p for p in (range(pos // self.P + 1) if pages is None else pages) if p >= 0]], hd)
                absk, big = np.abs(k).max(0), np.abs(v).max()
                A = R.attend_row(_abs_values(ref), table[b], x, hd, pos, scale, pages)[0]
                dx = 2.0 ** -17 * scale * (np.abs(x) @ absk)[:, None] + 2.0 ** -20
                tol = h * np.abs(o) + (r + 2 * dx + 2.0 ** -17) * A
                if self.dtype == "f16":
                    tol = tol + 2.0 ** -25 + (0 if alone else 2.0 ** -25 * len(v) * big)
                bad = np.abs(got - o) > tol
                assert not bad.any(), f"row {row} head {hd}: {np.abs(got - o)[bad].max()} over {tol[bad].min()}, {bad.sum()} of {bad.size}"
                if ld is not None:
                    off = np.abs(ld[row, hd * self.G:(hd + 1) * self.G] - l)
                    assert (off <= dx[:, 0] + 2.0 ** -20 * (1 + np.abs(l))).all(), (row, hd, off)
        # rows without a sequence stay as they were
        assert (od[self.real:] == 7.0).all() and (ld is None or (ld[self.real:] == 7.0).all())


def _abs_values(ref):
    c = R.Cache.__new__(R.Cache)
    c.__dict__.update(ref.__dict__)
    c.codes = ref.codes.copy()
    c.codes[:, :, 1] &= 0x7F
    return c
