"""What must not move: pages whose own values are appended again, and rows when what they do not see changes."""
import numpy as np
import pytest
import torch

from tests.q4_rig import DEV, D, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,lens,news", [(16, [0], [16]), (32, [5, 0, 16], [50, 33, 1]), (64, [63, 1], [70, 3]), (16, [3], [1])])
@pytest.mark.parametrize("scale", [1.0, 1e-3, 2.0 ** -20])
def test_values_that_were_read_back_are_appended_as_they_were(dtype, P, lens, news, scale):
    """Byte for byte: the largest element's code is 4 or 6 (or the scale is the least there is), so that it asks for the same scale again."""
    s = Step(lens, news, P=P, H=3, dtype=dtype, seed=P, spare=2)
    k, v = s.randn(s.T, s.H, D, scale=scale), s.randn(s.T, s.H, D, scale=scale / 3)
    k[:, :, 7] *= 30
    v[0] = 0.0
    s.cache.append(s.rows, k, v)
    held = s.cache.pages.clone()
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    s.cache.read(s.rows, ko, vo)
    assert not torch.equal(ko[: s.real], k[: s.real])
    s.cache.append(s.rows, ko, vo)
    assert torch.equal(s.cache.pages, held)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens,news", [([1000], [1]), ([975], [2]), ([973], [6]), ([965], [30]), ([960], [70])])
@pytest.mark.parametrize("gap", [14, 30, 60])
@pytest.mark.parametrize("how", ["row_from", "window"])
def test_a_hidden_page_of_large_values_costs_nothing(dtype, lens, news, gap, how):
    """The first page's values are 2^gap times as large as the others; some rows, or all, see what lies behind it only."""
    s = Step(lens, news, H=1, dtype=dtype, seed=gap)
    first = int(s.table[0, 0])
    s.cache.pages[:, :, :, 2112:] = 127 + (4 if dtype == "f16" else 10) - gap
    s.cache.pages[first, :, :, 2112:] = 127 + (4 if dtype == "f16" else 10)
    q = s.query(0.5)
    if how == "row_from":                                # every other row from the last, the only one where there is one
        row_from = np.array([16 if (s.real - 1 - r) % 2 == 0 else 0 for r in range(s.T)], dtype=np.int32)
        kw, blind = dict(row_from=row_from), [r for r in range(s.real) if row_from[r]]
    else:                                                # the last row sees 16 and on, those before it up to as many tokens more
        kw, blind = dict(window=s.pos[-1] - 15), [s.real - 1]
    out, lse = s.attend(q, **kw)
    s.check(q, out, lse, rows=sorted(set(list(range(0, s.real, 5)) + blind[-3:])), **kw)
    for other in (0, 127 - 96, 127 + 125):
        s.cache.pages[first, :, :, 2112:] = other
        again, ls = s.attend(q, **kw)
        assert torch.equal(again[blind], out[blind]) and torch.equal(ls[blind], lse[blind]), other
