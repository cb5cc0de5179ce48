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
