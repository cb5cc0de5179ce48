"""Reading back so many tokens that a wave takes two heads: any order, repeats, tokens that are none, even and odd numbers of heads."""
import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd as K
from tests import q4_ref as R
from tests.q4_rig import DEV, D, Step, i32, torch_type

pytestmark = pytest.mark.gpu


def _tokens(s, T, order, rng):
    """T sequences and positions among the step's tokens."""
    ends = [a + n for a, n in zip(s.lens, s.news)]
    seq = np.repeat(np.arange(len(ends)), ends)
    pos = np.concatenate([np.arange(e) for e in ends])
    if order == "in order":
        at = np.arange(T) % len(seq)
    elif order == "backwards":
        at = len(seq) - 1 - np.arange(T) % len(seq)
    elif order == "by chance":
        at = rng.integers(0, len(seq), T)
    else:                                                # pieces of up to 40 tokens, begun anywhere in a tile
        at = np.concatenate([b + np.arange(n) for b, n in zip(rng.integers(0, len(seq) - 40, T), rng.integers(1, 41, T))])[:T]
    return seq[at], pos[at]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,T", [(2, 32755), (3, 21841), (3, 22003), (5, 13121), (8, 8176), (8, 8177), (8, 9001)])
@pytest.mark.parametrize("order", ["in order", "backwards", "by chance", "in pieces"])
def test_read_many(dtype, H, T, order):
    """From ceil(T / 16) * H = 4096 on a wave has two heads; 8176 rows of 8 heads are the last that have one."""
    s = Step([700, 0, 301, 90], [1, 1, 3, 1], P=16 if H % 2 else 48, H=H, G=1, dtype=dtype, seed=H, exps=(-9, 15))
    rng = np.random.default_rng(T)
    seq, pos = _tokens(s, T, order, rng)
    for i, (b, p) in enumerate([(-1, 3), (4, 0), (0, -1), (1, 10 ** 6), (2 ** 31 - 1, 0), (0, 2 ** 31 - 1)]):     # no token there
        at = np.arange(37 + 5 * i, T, 1009)
        seq[at], pos[at] = b, p
    table = s.table.copy()
    table[2, 1], table[0, 3] = -1, s.NB                  # no block there
    rows = K.Q8Rows(i32(table), page_size=s.P, n_blocks=s.NB, n_rows=T, row_seq=i32(seq), row_pos=i32(pos))
    dt = torch_type(dtype)
    wide = torch.full((T, 2 * H + 1, D), 7.0, dtype=dt, device=DEV)
    s.cache.read(rows, wide[:, :H], wide[:, H + 1:])
    got = wide.double().cpu().numpy()
    assert (got[:, H] == 7.0).all()
    ref, (B, NP), top = s.ref(), table.shape, float(torch.finfo(dt).max)
    there = (seq >= 0) & (seq < B) & (pos >= 0) & (pos < NP * s.P)
    block = np.where(there, table[np.where(there, seq, 0), np.where(there, pos, 0) // s.P], -1)
    there &= (block >= 0) & (block < s.NB)
    assert there.any() and not there.all()
    for which, x in ((0, got[:, :H]), (1, got[:, H + 1:])):
        assert (x[~there] == 7.0).all()
        code, e = (a[block[there], :, which, pos[there] % s.P] for a in (ref.codes, ref.exps))
        assert np.array_equal(x[there], np.clip(R.number(code, np.repeat(e, 32, -1)), -top, top)), which
