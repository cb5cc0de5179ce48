"""The 8-bit paged cache on the GPU against its 64-bit definition (tests/q8_ref.py): page tables, appending, selection and
attention one by one at the sizes where they can go wrong, then together as a serving loop uses them."""
import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd as K
from tests import q8_ref as R
from tests import q8_rig as G
from tests.q8_rig import DEV, D, Step, i32

pytestmark = pytest.mark.gpu


# ---- page tables and slot maps ---------------------------------------------------------------------

def _map(lens, news, P, *, NP=None, T=None, Rn=None, free=None, count=None, NB=1000):
    B = len(lens)
    NP = NP or max(1, max(-(-(a + n) // P) for a, n in zip(lens, news)))
    T = T if T is not None else max(1, sum(news))
    rng = np.random.default_rng(B * 7 + P)
    table = rng.integers(0, NB, (B, NP))
    free = rng.permutation(NB).tolist() if free is None else free
    count = len(free) if count is None else count
    Rn = Rn or min(T, T // P + 2 * B)
    dt = i32(table)
    rows = K.Q8Rows(dt, page_size=P, n_blocks=NB, n_rows=T, max_runs=Rn)
    for t in (rows.kv_len, rows.row_start, rows.row_seq, rows.row_pos, rows.runs, rows.counts):
        t.fill_(77)
    rows.map(i32(lens), i32(news), i32(free), i32([count]))
    want = R.map_step(lens, news, table, free, count, P, T, Rn)
    for name, w in want.items():
        got = getattr(rows, name).cpu().numpy()
        assert np.array_equal(got, np.array(w).reshape(got.shape)), name
    assert np.array_equal(dt.cpu().numpy(), table)
    return want


@pytest.mark.parametrize("P", [16, 48, 256])
@pytest.mark.parametrize("lens,news", [
    ([0], [1]), ([15], [1]), ([16], [1]), ([17], [0]), ([0], [777]), ([5, 0, 31, 32, 100], [1, 1, 1, 1, 1]),
    ([0, 0, 9, 0, 0], [0, 3, 0, 500, 0]), ([1000, 3, 64], [300, 16, 15]), ([0] * 7, [0] * 7),
])
def test_map(P, lens, news):
    _map(lens, news, P, NP=90)
    _map(lens, news, P, NP=90, T=sum(news) + 29)


def test_map_of_many_sequences():
    rng = np.random.default_rng(3)
    for B, top in ((4096, 3), (1000, 40), (513, 200)):
        lens, news = rng.integers(0, 500, B), rng.integers(0, top, B)
        _map(lens.tolist(), news.tolist(), 16, NB=40000, T=int(news.sum()) + 5)


def test_map_that_does_not_fit_changes_nothing():
    assert _map([0, 0], [40, 10], 16, free=[3, 4, 5], count=3)["counts"][4] == 1      # four pages
    assert _map([0, 0], [40, 8], 16, free=[3, 4, 5, 6], count=3)["counts"][4] == 1
    assert _map([0, 0], [32, 8], 16, free=[3, 4, 5], count=9)["counts"] == [40, 3, 3, 0, 0]   # no more than the list holds
    assert _map([0, 0], [40, 10], 16, T=49)["counts"][4] == 2
    assert _map([0, 0], [40, 10], 16, Rn=3)["counts"][4] == 4
    assert _map([0, -1], [40, 10], 16)["counts"][4] == 8
    assert _map([0, 100], [4, 29], 16, NP=8)["counts"][4] == 8
    assert _map([0, 2 ** 31 - 1], [4, 2 ** 31 - 1], 16, NP=8, T=60)["counts"][4] == 8
    assert _map([0, 0], [4, 128], 16, NP=8, T=60)["counts"][4] == 2
    assert _map([0, 100], [64, 29], 16, NP=8, T=60, free=[1], count=-5)["counts"][4] & 8


# ---- appending -------------------------------------------------------------------------------------

def _append(s, k, v):
    ref = G.to_ref(s.cache, s.P)
    s.cache.append(s.rows, k, v)
    ref.append(s.runs, k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(s.cache.exps.cpu().numpy(), ref.exps)
    assert np.array_equal(s.cache.pages.cpu().numpy(), ref.bytes())
    assert np.array_equal(s.cache.means.cpu().numpy(), ref.means)
    assert np.array_equal(s.cache.mean_scales.cpu().numpy(), ref.mean_scales)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,lens,news", [
    (16, [0], [1]), (16, [15, 16, 0, 3], [1, 1, 1, 1]), (16, [0, 7, 30], [100, 9, 3]), (48, [0, 7, 47, 96], [100, 41, 1, 200]),
    (256, [0, 250, 17], [300, 20, 16]), (64, [5, 63], [1, 1]), (32, [20, 0], [12, 0]),
])
@pytest.mark.parametrize("scale", [1.0, 30.0, 1e-3])
def test_append(dtype, P, lens, news, scale):
    s = Step(lens, news, P=P, H=3, dtype=dtype, seed=P + len(lens), spare=2)
    k, v = s.randn(s.T, s.H, D, scale=scale), s.randn(s.T, s.H, D, scale=scale / 3)
    k[:, :, 5] *= 9
    _append(s, k, v)
    _append(s, k, v)                                     # the same once more: nothing moves


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_append_of_values_at_the_ends_of_the_range(dtype):
    s = Step([0, 3, 0, 0, 5], [16, 6, 1, 16, 2], dtype=dtype, seed=5)
    k, v = s.randn(s.T, s.H, D), s.randn(s.T, s.H, D)
    top = torch.finfo(k.dtype).max
    k[0, 0, 0], k[1, 0, 1], k[2, 0, 2], k[3, 1, 7] = float("nan"), float("inf"), float("-inf"), top
    v[0, 1, 3], v[2, 0, 4], v[5, 0, 9] = float("inf"), float("nan"), -top
    k[16:22, 0], v[16:22, 1] = 0.0, float("nan")          # all zeros into a page that holds something; all NaN
    k[22], v[22] = float("inf"), 0.0                       # nothing finite
    k[23:39] *= torch.finfo(k.dtype).tiny                  # the smallest numbers
    v[23:39] = torch.finfo(v.dtype).smallest_normal / 4
    _append(s, k, v)


def test_append_from_strided_rows():
    s = Step([0, 3], [40, 9], dtype="f16", H=2, seed=6)
    qkv = s.randn(s.T, 2 * s.H + 3, D)
    _append(s, qkv[:, :2], qkv[:, 3:5])
    s = Step([9], [1], H=2, seed=6)
    one = s.randn(1, 8, D)
    _append(s, one[:, :2], one[:, 4:6])


def test_append_leaves_out_runs_that_cannot_be():
    s = Step([0, 0, 0, 0, 0, 0, 0, 0], [4] * 8, seed=7)
    T = s.T
    for i, bad in enumerate(([s.NB, 0, 0, 4], [-1, 4, 0, 4], [1, 8, 13, 4], [1, 8, -1, 4], [1, 30, 0, 4], [1, -1, 0, 4], [1, 8, 0, 0])):
        s.runs[i] = bad
    assert T == 32
    s.rows.runs.copy_(i32(s.runs))
    _append(s, s.randn(T, s.H, D), s.randn(T, s.H, D))


# ---- selection -------------------------------------------------------------------------------------

def _select(s, q, k, sink=0, recent=0, rows=None, table=None):
    s.cache.c.sink_pages, s.cache.c.recent_pages = sink, recent
    sel = torch.full((s.T, s.H, k), -9, dtype=torch.int32, device=DEV)
    s.cache.select(s.rows, q, sel, s.cache.workspace(s.rows, select=True))
    got, ref, qd = sel.cpu().numpy(), G.to_ref(s.cache, s.P), q.double().cpu().numpy()
    table = s.table if table is None else table
    for r in (range(s.real) if rows is None else rows):
        for h in range(s.H):
            want = R.select_row(ref, table[s.seq[r]], qd[r, h * s.G:(h + 1) * s.G], h, s.pos[r], k, sink, recent, s.NB)
            assert got[r, h].tolist() == want, (r, h)
    assert (got[s.real:] == -9).all()
    return sel


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,lens,news,k,sink,recent", [
    (16, [0], [1], 1, 0, 0), (16, [1000, 3, 499], [1, 1, 1], 8, 0, 0), (16, [1000, 3, 499], [1, 1, 1], 8, 1, 2),
    (32, [3000, 900], [3, 1], 17, 0, 1), (48, [2000], [40], 5, 2, 3), (16, [9000, 40], [1, 20], 64, 0, 0),
    (16, [20000], [1], 700, 3, 4), (64, [100, 100], [1, 1], 64, 0, 0), (16, [0, 260], [33, 17], 4, 4, 0), (16, [300], [1], 4, 0, 4),
])
def test_select(dtype, P, lens, news, k, sink, recent):
    s = Step(lens, news, P=P, H=2, G=3 if k == 17 else 4, dtype=dtype, seed=k, spare=3)
    _select(s, s.query(), k, sink, recent)


@pytest.mark.parametrize("pages,k", [(16383, 100), (16385, 2048), (65536, 1000)])
def test_select_among_many_pages(pages, k):
    """Many pages share blocks here, so that scores are equal by the hundred and the lowest pages decide."""
    s = Step([0], [1], P=16, H=1, G=8, seed=pages, max_pages=pages, blocks=300)
    s.pos, s.lens = [pages * 16 - 3], [pages * 16 - 3]
    s.table[:] = np.random.default_rng(1).integers(0, 300, (1, pages))
    s.rows.page_table.copy_(i32(s.table))
    s.rows.row_pos.copy_(i32(s.pos))
    s.rows.kv_len.copy_(i32([pages * 16 - 2]))
    _select(s, s.query(), k)


@pytest.mark.parametrize("H", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("lens,news,max_pages", [([900, 2100], [1, 3], None), ([500, 3, 333] * 20, [10] * 60, None),
                                                 ([2900, 700] * 10, [40, 1] * 10, 800)])
def test_select_of_any_number_of_heads_for_few_rows_and_many(H, lens, news, max_pages):
    s = Step(lens, news, P=16, H=H, G=2, seed=H, max_pages=max_pages)
    _select(s, s.query(), 9, 1, 1, rows=range(0, s.real, 1 + s.real // 12))


def test_select_with_equal_scores_bad_blocks_and_queries_that_are_no_numbers():
    s = Step([800, 800, 800], [1, 1, 1], seed=9)
    q = s.query()
    q[0, 0] = float("nan")
    q[1] = 0.0
    q[2, 5, 3] = float("inf")
    _select(s, q, 10)
    s.cache.means.fill_(3)
    s.cache.mean_scales.fill_(0.5)
    _select(s, s.query(), 10, 0, 1)
    table = s.table.copy()
    table[0, 3], table[1, :45], table[2, 7] = -1, s.NB, 2 ** 31 - 1
    s.rows.page_table.copy_(i32(table))
    _select(s, s.query(), 10, table=table)


# ---- attention -------------------------------------------------------------------------------------

ROWS = [
    ([0], [1]), ([1], [1]), ([14], [1]), ([15], [1]), ([16], [1]), ([31, 0, 700], [1, 1, 1]), ([2000], [1]), ([5000, 1, 37], [1, 0, 1]),
    ([0, 0], [2, 1]), ([100], [2]), ([300, 4], [4, 3]), ([0], [40]), ([37, 500], [70, 5]), ([0, 11, 0], [200, 1, 33]),
    ([1500], [33]), ([0, 90], [0, 65]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,H,Gq", [(16, 2, 4), (48, 1, 7), (32, 3, 1), (256, 1, 8)])
@pytest.mark.parametrize("lens,news", ROWS)
def test_attend(dtype, P, H, Gq, lens, news):
    s = Step(lens, news, P=P, H=H, G=Gq, dtype=dtype, seed=len(lens) + P, spare=0 if len(lens) > 1 else 1 if sum(news) > 1 else 0)
    q = s.query(2.0)
    out, lse = s.attend(q)
    rows = range(s.real) if s.real < 60 else sorted(set(list(range(0, s.real, 7)) + [s.real - 1]))
    s.check_attention(q, out, lse, rows=rows)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_long_and_ragged(dtype):
    s = Step([70000, 0, 12345, 3, 800], [1, 1, 1, 1, 1], P=32, H=2, G=5, dtype=dtype, seed=3)
    q = s.query(3.0)
    s.check_attention(q, *s.attend(q))
    s = Step([30000, 0, 2345, 3], [3, 1, 2, 4], P=16, H=1, G=8, dtype=dtype, seed=4)
    q = s.query(3.0)
    s.check_attention(q, *s.attend(q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Gq", [2, 3, 5, 6])
@pytest.mark.parametrize("lens,news", [([0, 37, 5], [290, 41, 1]), ([9000], [70])])
def test_attend_many_rows_of_any_group(dtype, Gq, lens, news):
    s = Step(lens, news, P=32, H=2, G=Gq, dtype=dtype, seed=Gq, spare=1)
    q = s.query(2.0)
    s.check_attention(q, *s.attend(q), rows=sorted(set(list(range(0, s.real, 23)) + [s.real - 2, s.real - 1])))


def test_attend_many_short_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 60, 700).tolist()
    s = Step(lens, [1] * 700, H=2, G=2, seed=5, spare=0)
    q = s.query()
    s.check_attention(q, *s.attend(q), rows=range(0, 700, 9))
    s = Step(lens[:300], [2] * 300, H=2, G=2, seed=5)
    q = s.query()
    s.check_attention(q, *s.attend(q), rows=range(0, 600, 11))


def test_attend_keeps_pages_of_small_values_beside_a_page_of_large_ones():
    """f16: one page's values are 2^14 times as large as the others', and lies behind what most rows see."""
    for news in ([1], [30], [60]):
        s = Step([1000], news, dtype="f16", H=1, seed=31)
        s.cache.exps[:, :, 1] = -9
        s.cache.exps[int(s.table[0, (999 + news[0]) // 16]), :, 1] = 5
        q = s.query(0.5)
        out, lse = s.attend(q)
        s.check_attention(q, out, lse)
        # rows in front of that page: each of up to 1060 weights is off by 2^-11, or, below 2^-14 of 2^-7, by 2^-25 of it, and the output by 2^-11
        ref = G.to_ref(s.cache, 16)
        first = s.pos.index(next(p for p in s.pos if p // 16 == (999 + news[0]) // 16))
        for r in range(0, first, 5):
            o, _ = R.attend_row(ref, s.table[0], q[r].double().cpu().numpy(), 0, s.pos[r], 1 / np.sqrt(128.0))
            big = np.abs(R.VALUES[ref.codes[s.table[0, : s.pos[r] // 16 + 1], 0, 1]]).max() * 2.0 ** -9
            got = out[r].double().cpu().numpy()
            assert np.abs(got - o).max() <= 2.0 ** -11 * np.abs(o).max() + (2.0 ** -11 + 2.0 ** -15) * big + 2.0 ** -25


@pytest.mark.parametrize("news", [[1, 1], [9, 30]])
def test_attend_with_one_logit_far_above_the_rest_and_scales_far_apart(news):
    for dtype in ("bf16", "f16"):
        s = Step([700, 90], news, dtype=dtype, seed=8)
        s.cache.exps.copy_(torch.randint(-14, -3, s.cache.exps.shape, generator=s.gen, device=DEV))
        q = s.query(8.0)
        s.check_attention(q, *s.attend(q))


def test_attend_strided_queries_no_lse_and_a_scale_of_its_own():
    s = Step([50, 90], [3, 1], seed=9)
    wide = s.randn(s.T, s.H * s.G + 4, D)
    q = wide[:, 1:1 + s.H * s.G]
    out, lse = s.attend(q)
    s.check_attention(q, out, lse)
    again, none = s.attend(q, lse=False)
    assert none is None and torch.equal(again, out)
    s.cache.c.softmax_scale = 2.0 / np.sqrt(128.0)
    twice, l2 = s.attend(q)
    s.cache.c.softmax_scale = 0.0
    want, l1 = s.attend((q.float() * 2).to(q.dtype))      # (twice a number is exact)
    assert torch.allclose(l2, l1, rtol=1e-6, atol=1e-6)
    assert (twice.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()


@pytest.mark.parametrize("news", [[1, 1, 1], [5, 2, 20]])
def test_attend_keeps_bad_blocks_and_hidden_tokens_out(news):
    s = Step([300, 40, 0], news, seed=10)
    table = s.table.copy()
    table[0, 2], table[0, 5], table[2, 0] = -1, s.NB, -2 ** 31
    s.rows.page_table.copy_(i32(table))
    q = s.query()
    s.check_attention(q, *s.attend(q), table=table)
    # what lies behind a sequence's last token, and in pages that nobody reads, has no influence
    before = s.attend(q)
    ref_places = R.tile_places(16)
    end = 300 + news[0]
    last = int(table[0, (end - 1) // 16])
    for t in range(end % 16, 16) if end % 16 else ():
        flat = s.cache.pages.view(s.NB, s.H, -1)
        flat[last][:, torch.from_numpy(ref_places[0][t]).to(DEV)] = 0x7E
        flat[last][:, torch.from_numpy(ref_places[1][t]).to(DEV)] = 0x7E
    after = s.attend(q)
    assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1])


def test_a_row_that_is_no_number_stays_alone():
    s = Step([300, 40], [5, 6], seed=11)
    q = s.query()
    good, glse = s.attend(q)
    bad = q.clone()
    bad[3, 2, 7] = float("nan")
    out, lse = s.attend(bad)
    assert torch.isnan(out[3, 2]).all() and torch.isnan(lse[3, 2])
    out[3, 2], lse[3, 2] = good[3, 2], glse[3, 2]
    assert torch.equal(out, good) and torch.equal(lse, glse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,lens,news,k", [
    (16, [0], [1], 1), (16, [1000, 3, 499], [1, 1, 1], 8), (32, [3000, 900], [3, 1], 17), (48, [2000], [40], 5),
    (16, [20000], [1], 700), (256, [5000], [2], 3), (16, [100] * 90, [6] * 90, 3),
])
def test_attend_selected(dtype, P, lens, news, k):
    s = Step(lens, news, P=P, H=2, G=3 if k == 17 else 4, dtype=dtype, seed=k, spare=2)
    q = s.query(2.0)
    sel = _select(s, q, k, 0, 1, rows=[])
    out, lse = s.attend(q, sel)
    s.check_attention(q, out, lse, sel, rows=range(0, s.real, 1 + s.real // 40))
    # every page selected is all of them
    if k == 1:
        full, flse = s.attend(q)
        assert torch.allclose(lse[:s.real], flse[:s.real], rtol=1e-6, atol=1e-6)


def test_attend_selected_pages_that_are_none():
    s = Step([400, 400, 9], [1, 1, 1], seed=12)
    q = s.query()
    sel = torch.full((3, s.H, 6), -1, dtype=torch.int32, device=DEV)
    sel[0, 0, :3] = i32([2, 9, 25])
    sel[0, 1, :4] = i32([25, 0, 3, 1])
    sel[1, 0, :2] = i32([5, 10 ** 6])                     # a page beyond the table is not visible
    sel[2, :, 0] = 0
    out, lse = s.attend(q, sel)
    sel[1, 0, 1] = -1
    s.check_attention(q, out, lse, sel)


# ---- streams, graphs, workspaces, the whole ----------------------------------------------------------

def test_calls_on_two_streams_with_a_workspace_each():
    a, b = Step([9000, 40], [1, 1], seed=13), Step([5000, 700, 3], [7, 1, 2], dtype="f16", seed=14)
    qa, qb = a.query(), b.query()
    wa, wb = a.attend(qa), b.attend(qb)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    wsa, wsb = a.cache.workspace(a.rows), b.cache.workspace(b.rows)
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        with torch.cuda.stream(sa):
            got.append((a.attend(qa, ws=wsa), wa))
        with torch.cuda.stream(sb):
            got.append((b.attend(qb, ws=wsb), wb))
    torch.cuda.synchronize()
    for (o, l), (wo, wl) in got:
        assert torch.equal(o, wo) and torch.equal(l, wl)
    # every call leaves the workspace ready: the counters at its start are zero again
    assert int(wsa[:2048].abs().max()) == 0 and int(wsb[:2048].abs().max()) == 0


class Server:
    """A serving loop: requests of growing length, their pages and blocks, one layer."""

    def __init__(self, B, NP, NB, T, P=16, H=2, Gq=4, dtype="bf16", k=6):
        self.P, self.H, self.G, self.NB, self.k = P, H, Gq, NB, k
        self.dt = G.torch_type(dtype)
        self.cache = K.Q8Cache(n_blocks=NB, n_q_heads=H * Gq, n_kv_heads=H, page_size=P, kv_dtype=self.dt, sink_pages=1, recent_pages=1,
                               device=DEV)
        self.rows = K.Q8Rows(torch.full((B, NP), -1, dtype=torch.int32, device=DEV), page_size=P, n_blocks=NB, n_rows=T)
        self.seq_len, self.n_new = i32([0] * B), i32([0] * B)
        self.free = i32(np.random.default_rng(0).permutation(NB))
        self.count = i32([NB])
        self.q = torch.zeros((T, H * Gq, D), dtype=self.dt, device=DEV)
        self.kn, self.vn = (torch.zeros((T, H, D), dtype=self.dt, device=DEV) for _ in range(2))
        self.sel = torch.full((T, H, k), -1, dtype=torch.int32, device=DEV)
        self.out, self.sparse = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.lse = torch.zeros((T, H * Gq), device=DEV)
        self.ws, self.ws_sel = self.cache.workspace(self.rows), self.cache.workspace(self.rows, select=True)

    def step(self):
        self.rows.map(self.seq_len, self.n_new, self.free, self.count)
        self.cache.append(self.rows, self.kn, self.vn)
        self.cache.attend(self.rows, self.q, self.out, self.ws, lse=self.lse)
        self.cache.select(self.rows, self.q, self.sel, self.ws_sel)
        self.cache.attend(self.rows, self.q, self.sparse, self.ws, sel_pages=self.sel)
        self.seq_len.copy_(self.rows.kv_len)
        self.count.copy_(self.rows.counts[3:4])

    def results(self):
        return [t.clone() for t in (self.out, self.lse, self.sel, self.sparse, self.cache.pages, self.cache.exps, self.cache.means,
                                    self.rows.page_table, self.rows.kv_len, self.count)]


def _feed(server, i, news):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000 + i)
    for t in (server.q, server.kn, server.vn):
        t.copy_(torch.randn(t.shape, generator=g, device=DEV))
    server.n_new.copy_(i32(news))


def test_serving_steps_together():
    """Prompts, then single tokens, then drafts with some requests resting: every step against the definition."""
    B, NP, NB, T, P = 3, 30, 80, 150, 16
    s = Server(B, NP, NB, T)
    table, ref = np.full((B, NP), -1), R.Cache(NB, s.H, P)
    lens, count, free = [0] * B, NB, s.free.cpu().tolist()
    plan = [[100, 0, 37], [1, 1, 1], [1, 9, 1], [0, 3, 2], [60, 1, 60], [1, 1, 1], [2, 0, 2]]
    for i, news in enumerate(plan):
        _feed(s, i, news)
        s.step()
        want = R.map_step(lens, news, table, free, count, P, T, s.rows.max_runs)
        lens, count = want["kv_len"], want["counts"][3]
        ref.append(want["runs"], s.kn.double().cpu().numpy(), s.vn.double().cpu().numpy())
        assert np.array_equal(s.rows.page_table.cpu().numpy(), table) and s.rows.counts.cpu().tolist() == want["counts"]
        assert np.array_equal(s.cache.pages.cpu().numpy(), ref.bytes()) and np.array_equal(s.cache.exps.cpu().numpy(), ref.exps)
        q, sel = s.q.double().cpu().numpy(), s.sel.cpu().numpy()
        for r in range(0, want["counts"][0], 5):
            b, pos = want["row_seq"][r], want["row_pos"][r]
            for h in range(s.H):
                x = q[r, h * s.G:(h + 1) * s.G]
                pages = R.select_row(ref, table[b], x, h, pos, s.k, 1, 1, NB)
                assert sel[r, h].tolist() == pages, (i, r, h)
                for got, which in ((s.out, None), (s.sparse, pages)):
                    o, _ = R.attend_row(ref, table[b], x, h, pos, 1.0 / np.sqrt(128.0), which)
                    g = got[r, h * s.G:(h + 1) * s.G].double().cpu().numpy()
                    # half a step of bf16 each for the output and for P, with |v| below 5 in any average
                    assert np.abs(g - o).max() <= 2.0 ** -8 * (np.abs(o).max() + 5.0), (i, r, h)


def test_steps_in_a_graph_are_those_outside():
    """One captured step, replayed while the requests grow, against the same steps called one by one; the program's own work
    and synchronisations lie between the replays."""
    news = [1, 2, 1, 0]
    a, b = (Server(4, 40, 120, 6) for _ in range(2))
    for s in (a, b):
        for i in range(3):
            _feed(s, i, news)
            s.step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.step()
    for i in range(3, 40):
        for s in (a, b):
            _feed(s, i, [1, i % 3, 1, i % 2])
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x, y), i
        scratch = torch.randn(1 << 20, device=DEV).sum()
        assert torch.isfinite(scratch)


def test_results_do_not_change_from_call_to_call():
    s = Step([40000, 0, 1234, 3], [1, 1, 1, 1], H=2, G=5, seed=15)
    q = s.query()
    first = s.attend(q)
    for _ in range(20):
        o, l = s.attend(q)
        assert torch.equal(o, first[0]) and torch.equal(l, first[1])


def test_one_workspace_for_selections_and_attention_of_different_sizes():
    """A workspace that is large enough for all of them serves one call after another, whatever ran in it before."""
    steps = [Step([9000, 40], [1, 1], seed=21), Step([600, 700], [40, 9], dtype="f16", seed=22), Step([5000], [3], P=32, G=8, seed=23)]
    need = max(t.numel() for s in steps for t in (s.cache.workspace(s.rows), s.cache.workspace(s.rows, select=True)))
    ws = torch.zeros(need, dtype=torch.int32, device=DEV)
    qs = [s.query() for s in steps]
    alone = [(s.attend(q), _select(s, q, 9, 1, 1, rows=[])) for s, q in zip(steps, qs)]
    for _ in range(3):
        for s, q, (want, sel) in zip(steps, qs, alone):
            got = torch.full_like(sel, -9)
            s.cache.select(s.rows, q, got, ws)
            out, lse = s.attend(q, ws=ws)
            assert torch.equal(got, sel) and torch.equal(out, want[0]) and torch.equal(lse, want[1])
            o2, l2 = s.attend(q, sel=got, ws=ws)
            s.check_attention(q, o2, l2, got, rows=[0, s.real - 1])
    assert int(ws[:2048].abs().max()) == 0
