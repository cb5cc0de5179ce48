"""Attention of the 4-bit cache with caps, biases, windows, documents and prefixes in every layout that the query rows can have: copies of them
in 16 columns, up to four groups of 16, waves with rows of their own; contexts that one workgroup has and such as are joined."""
import numpy as np
import pytest

from tests.q4_rig import Step

pytestmark = pytest.mark.gpu

# columns of a sequence, on the average: 4, 8, 12, 21, 24, 32, 48, 56, 64, 96, 112, 128, 160, 256
FORMS = [([2500, 40], [1, 1], 4), ([1700, 3], [2, 2], 4), ([3100, 0, 17], [3, 3, 3], 4), ([900, 1333, 7], [3, 3, 3], 7), ([3000, 5], [6, 6], 4),
         ([2000, 60], [4, 4], 8), ([2500, 40], [12, 12], 4), ([2000], [8], 7), ([1200, 100], [64, 64], 1), ([1800, 0], [24, 24], 4), ([700, 30], [16, 16], 7),
         ([1500], [16], 8), ([0, 1100], [40, 40], 4), ([900], [64], 4)]
SCORES = [dict(softcap=30.0), dict(softcap=400.0), dict(slopes=True), dict(softcap=20.0, slopes=True), dict(softcap=90.0, slopes=True, window=700),
          dict(softcap=5.0, docs=333), dict(slopes=True, docs=77, prefix=True), dict(softcap=50.0, slopes=True, prefix=True)]
WEIGHTS = 2.0 ** -16


def _slopes(n):
    return np.array([2.0 ** (-8 * (i + 1) / n) * (-1 / 64 if i == 3 else 1) for i in range(n)], dtype=np.float32)


def _make(s, kw, rng):
    made = {n: kw[n] for n in ("softcap", "window") if n in kw}
    if "slopes" in kw:
        made["slopes"] = _slopes(s.H * s.G)
    if "docs" in kw:
        made["row_from"] = np.array([p // kw["docs"] * kw["docs"] for p in s.pos] + [0] * (s.T - s.real), dtype=np.int32)
    if "prefix" in kw:
        made["prefix_len"] = rng.integers(0, 1 + max(s.lens) + 20, len(s.lens)).astype(np.int32)
    return made


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kw", SCORES, ids=str)
@pytest.mark.parametrize("lens,news,Gq", FORMS)
def test_scores_of_all_kinds_in_every_layout(dtype, kw, lens, news, Gq):
    s = Step(lens, news, P=48 if Gq == 7 else 16, H=2, G=Gq, dtype=dtype, seed=Gq + len(kw))
    q = s.query(2.0)
    made = _make(s, kw, np.random.default_rng(Gq))
    out, lse = s.attend(q, **made)
    s.check(q, out, lse, rows=sorted({0, s.real - 1} | set(range(0, s.real, 1 + s.real // 12))), weights=WEIGHTS, **made)


@pytest.mark.parametrize("seed", range(48))
def test_scores_and_rows_by_chance(seed):
    rng = np.random.default_rng(1000 + seed)
    B = int(rng.choice([1, 2, 5, 30]))
    top = {1: 20000, 2: 9000, 5: 3000, 30: 600}[B]
    lens = np.exp(rng.uniform(0, np.log(top), B)).astype(int).tolist()
    most = int(rng.choice([1, 2, 4, 8, 12, 20, 40, 100])) if B < 30 else int(rng.choice([1, 3, 9]))
    news = rng.integers(1, most + 1, B).tolist()
    s = Step(lens, news, P=int(rng.choice([16, 48, 128])), H=int(rng.choice([1, 3])), G=int(rng.choice([1, 2, 4, 5, 7, 8])), seed=seed,
             dtype=["bf16", "f16"][seed % 2], spare=seed % 3)
    q = s.query(2.0)
    kw = {}
    if seed % 4:
        kw["softcap"] = float(np.exp(rng.uniform(np.log(3), np.log(63)) if seed % 4 < 3 else rng.uniform(np.log(65), np.log(3000))))
    if seed % 3 != 1:
        kw["slopes"] = True
    mask = ["", "window", "docs", "prefix"][int(rng.integers(0, 4))]
    if mask:
        kw[mask] = int(rng.integers(1, top))
    made = _make(s, kw, rng)
    s.check(q, *s.attend(q, **made), rows=sorted(set(rng.integers(0, s.real, 16).tolist())), weights=WEIGHTS, **made)
