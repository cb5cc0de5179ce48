"""The 8-bit paged cache on the GPU where values, scales and scores lie far apart: what one page holds must not cost
another page's tokens their weights, and what a row does not see must not reach it.  Against tests/q8_ref.py."""
import math

import numpy as np
import pytest
import torch

from tests import q8_ref as R
from tests import q8_rig as G
from tests.q8_rig import D, Step, i32

pytestmark = pytest.mark.gpu

# (tokens before, new ones) of sequences with 4 query heads a KV head and pages of 16: rows of one page, then rows of the next
# one, which is the second tile of the same pair.  2, 6 and 30 rows take one and two groups of columns and the rows' form.
SPLIT = [([975], [2]), ([15], [2]), ([973], [6]), ([12], [6]), ([965], [30]), ([0], [40])]


def _bound(s, ref, row, head, q, scale, r):
    """(out, lse, bound of out) of a row and head in 64 bits.  With A = sum p |v| / sum p: half a step of the type of the
    output, `r` of A for the weights' own rounding, twice the logits' error (128 products and their sums in fp32: 2^-17 sum |q k|
    scale; exponent and maximum 2^-20) and the sums' and joins' 2^-17 of A, and half of f16's least step."""
    h = torch.finfo(G.torch_type(s.dtype)).eps / 2
    b, pos = s.seq[row], s.pos[row]
    x = q[row, head * s.G:(head + 1) * s.G].double().cpu().numpy()
    o, l = R.attend_row(ref, s.table[b], x, head, pos, scale)
    A = R.attend_row(G._abs_values(ref), s.table[b], x, head, pos, scale)[0]
    k, _ = ref.kv(s.table[b][: pos // s.P + 1], head)
    dx = 2.0 ** -17 * scale * (np.abs(x) @ np.abs(k).max(0))[:, None] + 2.0 ** -20
    return o, l, h * np.abs(o) + (r + 2 * dx + 2.0 ** -17) * A + (2.0 ** -25 if s.dtype == "f16" else 0.0)


@pytest.mark.parametrize("lens,news", SPLIT)
@pytest.mark.parametrize("gap", [14, 20, 24, 28, 32])
def test_a_later_page_of_large_values_costs_the_rows_before_it_nothing(lens, news, gap):
    """f16: the page behind the first rows' holds values up to 2^15, 2^gap times as large as all the others."""
    s = Step(lens, news, dtype="f16", H=2, seed=gap)
    s.cache.exps[:, :, 1] = 6 - gap
    s.cache.exps[int(s.table[0, lens[0] // 16 + 1]), :, 1] = 6
    q = s.query(0.5)
    out, lse = s.attend(q)
    ref = G.to_ref(s.cache, s.P)
    for row in range(s.real):
        for head in range(s.H):
            o, l, tol = _bound(s, ref, row, head, q, 1.0 / math.sqrt(D), 2.0 ** -11)
            got = out[row, head * s.G:(head + 1) * s.G].double().cpu().numpy()
            assert (np.abs(got - o) <= tol).all(), (row, head, np.abs(got - o).max(), tol.min())


@pytest.mark.parametrize("lens,news", [([1000], [1]), ([975], [2]), ([973], [6]), ([965], [30])])
@pytest.mark.parametrize("gap", [20, 28, 36])
def test_a_visible_page_of_large_values_and_no_weight_costs_the_others_nothing(lens, news, gap):
    """f16: a page of values 2^gap times as large, whose keys give it weights below 2^-100 of the others'."""
    s = Step(lens, news, dtype="f16", H=1, seed=gap + 1)
    block = int(s.table[0, 3])
    s.cache.exps[:, :, 1] = 7 - gap
    s.cache.exps[block, :, 1] = 7
    q = s.query(0.5)
    q[..., 0] = 8.0
    key, _ = R.tile_places(16)
    s.cache.exps[block, :, 0] = -2
    s.cache.pages.view(s.NB, s.H, -1)[block, 0, torch.from_numpy(key[:, 0]).to(G.DEV)] = 0xFE           # -448 * 2^-2: logits of -79
    out, _ = s.attend(q)
    ref = G.to_ref(s.cache, s.P)
    for row in range(s.real):
        o, l, tol = _bound(s, ref, row, 0, q, 1.0 / math.sqrt(D), 2.0 ** -11)
        # (2^-100 of 2^16 is nothing)
        got = out[row].double().cpu().numpy()
        assert (np.abs(got - o) <= tol).all(), (row, np.abs(got - o).max(), tol.min())


# ---- the top of the range: magnitudes above 448 * 2^119, whose codes stand for numbers up to 448 * 2^120

@pytest.mark.parametrize("lens,news", [([1000], [1])] + SPLIT)
def test_values_at_the_top_of_the_range_are_numbers(lens, news):
    """bf16: every value of the second page of a pair, which the first rows do not see, is of the largest scale."""
    s = Step(lens, news, H=2, seed=41)
    block = int(s.table[0, (lens[0] // 16 + 1) if news[0] > 1 else 5])
    s.cache.exps[block, :, 1] = 120
    q = s.query(0.25)
    s.check_attention(q, *s.attend(q))


@pytest.mark.parametrize("lens,news", SPLIT)
def test_hidden_keys_at_the_top_of_the_range_reach_nothing(lens, news):
    s = Step(lens, news, H=2, seed=42)
    s.cache.exps[int(s.table[0, lens[0] // 16 + 1])] = 120
    q = s.query(0.25)
    before = [r for r in range(s.real) if s.pos[r] // 16 == lens[0] // 16]
    s.check_attention(q, *s.attend(q), rows=before)


@pytest.mark.parametrize("lens,news", [([70000], [1]), ([70000], [2]), ([9000], [6]), ([6000], [40])])
@pytest.mark.parametrize("growing", [False, True])
def test_sums_of_many_values_at_the_top_of_the_range_are_numbers(lens, news, growing):
    """Every value is between 104 and 240 times 2^120, that is below bf16's largest number, and so is their mean; with `growing` all
    tokens but the first few have e^5 times the weight of those, which is when weights are largest."""
    s = Step(lens, news, H=1, seed=43)
    s.cache.exps[:, :, 1] = 120
    _, val = R.tile_places(16)
    at = torch.from_numpy(val.ravel()).to(G.DEV)
    flat = s.cache.pages.view(s.NB, s.H, -1)
    flat[:, :, at] = torch.randint(0x6D, 0x78, (s.NB, s.H, at.numel()), generator=s.gen, device=G.DEV, dtype=torch.uint8)
    q = s.query(0.1)
    if growing:
        key, _ = R.tile_places(16)
        s.cache.exps[:, :, 0] = -5
        q[..., 0] = 4.0
        flat[:, :, torch.from_numpy(key[:, 0]).to(G.DEV)] = 0x7E                            # 448 * 2^-5: logits of 4.95
        flat[int(s.table[0, 0])][:, torch.from_numpy(key[:, 0]).to(G.DEV)] = 0
    out, lse = s.attend(q)
    ref = G.to_ref(s.cache, s.P)
    for row in range(0, s.real, 5):
        o, l, tol = _bound(s, ref, row, 0, q, 1.0 / math.sqrt(D), 2.0 ** -8)
        got = out[row].double().cpu().numpy()
        assert (np.abs(got - o) <= tol).all(), (row, got.max(), o.max())


@pytest.mark.parametrize("news", [[40], [1]])
def test_what_is_appended_at_the_ends_of_the_range_is_attended_to(news):
    """Tokens with bf16's largest number, with infinities and NaN beside it, behind ordinary ones."""
    s = Step([0] if news[0] > 1 else [39], news, H=2, seed=44)
    s.cache.exps.zero_()
    top = torch.finfo(torch.bfloat16).max
    T = 40
    full = s if news[0] > 1 else Step([0], [40], H=2, seed=44)
    k, v = full.randn(T, 2, D), full.randn(T, 2, D)
    v[20, 0, 3], v[21, 0, 4], v[22, 0, 5], v[39, 1, 7] = top, float("inf"), float("nan"), -top
    full.cache.append(full.rows, k, v)
    if full is not s:
        for b, c in zip(s.table[0], full.table[0]):
            for name in ("pages", "exps"):
                getattr(s.cache, name)[int(b)] = getattr(full.cache, name)[int(c)]
    q = s.query(0.25)
    s.check_attention(q, *s.attend(q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale,exp", [(1e-25, R.EXP_MIN), (1e6, 120)])
@pytest.mark.parametrize("lens,news", [([0], [1]), ([1000], [1])] + SPLIT)
def test_scales_that_leave_nothing_of_the_logits(dtype, scale, exp, lens, news):
    """softmax_scale = 1e-25 beside keys of the least scale (as pages of zeros have it), or 1e6 beside those of the largest and queries
    of 0: every logit is 0 in 32 bits, and every row the mean of the values that it sees.  All weights are the same power of two,
    so that an output is off by half a step of its type, 2^-17 of A for the sums, and what rounding 1/l costs."""
    s = Step(lens, news, dtype=dtype, H=2, seed=51, softmax_scale=scale)
    for page in (0, (lens[0] + news[0] - 1) // 16):
        s.cache.exps[int(s.table[0, page]), :, 0] = exp
    q = s.query(1.0 if scale < 1.0 else 0.0)
    out, lse = s.attend(q)
    ref = G.to_ref(s.cache, s.P)
    h = torch.finfo(G.torch_type(dtype)).eps / 2
    for row in range(s.real):
        n = s.pos[row] + 1
        for head in range(s.H):
            _, v = ref.kv(s.table[0][: (n - 1) // 16 + 1], head)
            o, A = v[:n].mean(0), np.abs(v[:n]).mean(0)
            got = out[row, head * s.G:(head + 1) * s.G].double().cpu().numpy()
            assert (np.abs(got - o) <= h * np.abs(o) + 2.0 ** -16 * A + (2.0 ** -25 if dtype == "f16" else 0.0)).all(), (row, head)
            assert np.abs(lse[row, head * s.G:(head + 1) * s.G].cpu().numpy() - math.log(n)).max() <= 2.0 ** -20 * (1 + math.log(n)), (row, head)


# ---- scores

@pytest.mark.parametrize("pages", [60, 1500])
def test_scores_of_minus_zero_are_those_of_zero(pages):
    """Pages whose scale is 0 score 0 whatever the sign of their product: a tie, which the lower page wins."""
    s = Step([pages * 16 - 2], [1], H=2, seed=61)
    s.cache.mean_scales.zero_()
    q = s.query()
    sel = torch.full((1, s.H, 9), -9, dtype=torch.int32, device=G.DEV)
    s.cache.select(s.rows, q, sel, s.cache.workspace(s.rows, select=True))
    assert sel.cpu().tolist() == [[list(range(9))] * s.H]


@pytest.mark.parametrize("H,lens,news", [(2, [900, 0, 333], [1, 3, 20]), (5, [400] * 9, [1, 2, 3, 16, 17, 1, 40, 1, 5])])
def test_selection_needs_sequences_and_positions_of_the_rows_only(H, lens, news):
    """Rows that a caller has filled without kv_len and row_start, with another selection's scores in the workspace."""
    s = Step(lens, news, H=H, seed=62)
    ws = s.cache.workspace(s.rows, select=True)
    want, got = (torch.full((s.T, H, 7), -9, dtype=torch.int32, device=G.DEV) for _ in range(2))
    q = s.query()
    s.cache.select(s.rows, q, want, ws)
    s.rows.row_start.fill_(10 ** 6)
    s.rows.kv_len.zero_()
    s.cache.select(s.rows, -q, got, ws)
    ref, qd = G.to_ref(s.cache, s.P), -q.double().cpu().numpy()
    for r in range(s.real):
        for h in range(H):
            assert got[r, h].tolist() == R.select_row(ref, s.table[s.seq[r]], qd[r, h * s.G:(h + 1) * s.G], h, s.pos[r], 7, 0, 0, s.NB), (r, h)
