"""The 4-bit paged cache on the GPU against its 64-bit definition (tests/q4_ref.py): appending, reading back and attention one by
one at the sizes and masks where they can go wrong, then together with the rotation as a serving loop uses them."""
import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd as K
from tests import q4_ref as R
from tests import q8_ref as R8
from tests.q4_rig import DEV, D, Step, i32, torch_type

pytestmark = pytest.mark.gpu


# ---- appending -------------------------------------------------------------------------------------

def _append(s, k, v):
    ref = s.ref()
    s.cache.append(s.rows, k, v)
    ref.append(s.runs, k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(s.cache.pages.cpu().numpy(), ref.bytes())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,lens,news", [
    (16, [0], [1]), (16, [15, 16, 0, 3], [1, 1, 1, 1]), (16, [0, 7, 30], [100, 9, 3]), (48, [0, 7, 47, 96], [100, 41, 1, 200]),
    (256, [0, 250, 17], [300, 20, 16]), (64, [5, 63], [1, 1]), (32, [20, 0], [12, 0]), (16, [1, 2, 3, 5], [2, 1, 4, 6]),
])
@pytest.mark.parametrize("scale", [1.0, 1e-3])
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
    k[16:22, 0], v[16:22, 1] = 0.0, float("nan")          # all zeros; all NaN
    k[22], v[22] = float("inf"), -0.0                      # nothing finite
    k[23:39] *= torch.finfo(k.dtype).tiny                  # the smallest numbers
    v[23:39] = torch.finfo(v.dtype).smallest_normal / 4
    k[39, 0, :32] = 7.0                                    # 7 is the largest that 2^0 takes
    k[39, 0, 32:64] = 7.03125
    k[39, 0, 64:72] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0])      # halves between codes
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
    for i, bad in enumerate(([s.NB, 0, 0, 4], [-1, 4, 0, 4], [1, 8, 13, 4], [1, 8, -1, 4], [1, 30, 0, 4], [1, -1, 0, 4], [1, 8, 0, 0])):
        s.runs[i] = bad
    s.rows.runs.copy_(i32(s.runs))
    _append(s, s.randn(s.T, s.H, D), s.randn(s.T, s.H, D))


# ---- reading back ----------------------------------------------------------------------------------

def _read(s, seq, pos, table=None):
    """The tokens (seq, pos), whatever they are: exact, or left as they were."""
    n = len(seq)
    table = s.table if table is None else table
    rows = K.Q8Rows(i32(table), page_size=s.P, n_blocks=s.NB, n_rows=n, row_seq=i32(seq), row_pos=i32(pos))
    dt = torch_type(s.dtype)
    wide = torch.full((n, 2 * s.H + 1, D), 7.0, dtype=dt, device=DEV)
    s.cache.read(rows, wide[:, :s.H], wide[:, s.H + 1:])
    got = wide.double().cpu().numpy()
    ref = s.ref()
    top = float(torch.finfo(dt).max)
    B, NP = np.asarray(table).shape
    assert (got[:, s.H] == 7.0).all()
    for i in range(n):
        block = table[seq[i]][pos[i] // s.P] if 0 <= seq[i] < B and 0 <= pos[i] < NP * s.P else -1
        for h in range(s.H):
            for which in (0, 1):
                x = got[i, h if which == 0 else s.H + 1 + h]
                if not 0 <= block < s.NB:
                    assert (x == 7.0).all(), i
                    continue
                t = pos[i] % s.P
                want = R.number(ref.codes[block, h, which, t], np.repeat(ref.exps[block, h, which, t], 32))
                assert np.array_equal(x, np.clip(want, -top, top)), (i, h, which)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P", [16, 48, 256])
def test_read(dtype, P):
    s = Step([100, 0, 37], [1, 1, 3], P=P, H=3, dtype=dtype, seed=P, exps=(-9, 14))
    rng = np.random.default_rng(P)
    ends = [101, 1, 40]
    seq = [b for b in range(3) for _ in range(ends[b])]
    pos = [p for b in range(3) for p in range(ends[b])]
    _read(s, seq, pos)                                    # whole contexts
    at = rng.integers(0, len(seq), 77)                    # any tokens, some of them twice
    _read(s, [seq[i] for i in at], [pos[i] for i in at])
    _read(s, [2], [39])


def test_read_at_the_ends_of_the_range_and_of_tokens_that_are_none():
    s = Step([40, 40], [1, 1], dtype="f16", seed=3, exps=(12, 16))         # up to 6 * 2^15: more than f16 has
    _read(s, [0, 0, -1, 1, 2, 1, 1, 0], [0, 40, 3, 7, 3, -1, 48, 41])
    table = s.table.copy()
    table[0, 1], table[1, 2], table[1, 0] = -1, s.NB, 2 ** 31 - 1
    _read(s, [0, 0, 1, 1, 1], [15, 16, 40, 0, 20], table)
    for e in ((-96, -94), (124, 126)):
        _read(Step([40], [1], seed=4, exps=e), [0] * 41, list(range(41)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_is_appended_is_read_back_rounded(dtype):
    s = Step([5, 0, 16], [50, 33, 1], P=32, H=2, dtype=dtype, seed=8, spare=3)
    k, v = s.randn(s.T, s.H, D), s.randn(s.T, s.H, D)
    s.cache.append(s.rows, k, v)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    s.cache.read(s.rows, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        code, e = R.quantise(x[:s.real].double().cpu().numpy())
        assert np.array_equal(y[:s.real].double().cpu().numpy(), R.number(code, np.repeat(e, 32, -1)))
        assert (y[s.real:] == 7.0).all()
    # once more from what came back: a fixed point
    before = s.cache.pages.clone()
    s.cache.append(s.rows, ko, vo)
    k2, v2 = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    s.cache.read(s.rows, k2, v2)
    assert torch.equal(k2, ko) and torch.equal(v2, vo) and before.shape == s.cache.pages.shape


# ---- attention -------------------------------------------------------------------------------------

ROWS = [
    ([0], [1]), ([1], [1]), ([14], [1]), ([15], [1]), ([16], [1]), ([127], [1]), ([128], [1]), ([31, 0, 700], [1, 1, 1]), ([2000], [1]),
    ([5000, 1, 37], [1, 0, 1]), ([0, 0], [2, 1]), ([100], [2]), ([300, 4], [4, 3]), ([0], [40]), ([37, 500], [70, 5]),
    ([0, 11, 0], [200, 1, 33]), ([1500], [33]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,H,Gq", [(16, 2, 4), (48, 1, 7), (32, 3, 1), (256, 1, 8), (16, 1, 3)])
@pytest.mark.parametrize("lens,news", ROWS)
def test_attend(dtype, P, H, Gq, lens, news):
    s = Step(lens, news, P=P, H=H, G=Gq, dtype=dtype, seed=len(lens) + P, spare=0 if len(lens) > 1 else 1 if sum(news) > 1 else 0)
    q = s.query(2.0)
    out, lse = s.attend(q)
    s.check(q, out, lse, rows=range(s.real) if s.real < 60 else sorted(set(list(range(0, s.real, 7)) + [s.real - 1])))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_long_and_ragged(dtype):
    s = Step([70000, 0, 12345, 3, 800], [1, 1, 1, 1, 1], P=32, H=2, G=5, dtype=dtype, seed=3)
    q = s.query(3.0)
    s.check(q, *s.attend(q))
    s = Step([30000, 0, 2345, 3], [3, 1, 2, 4], P=16, H=1, G=8, dtype=dtype, seed=4)
    q = s.query(3.0)
    s.check(q, *s.attend(q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Gq", [1, 2, 3, 5, 6, 8])
@pytest.mark.parametrize("lens,news", [([0, 37, 5], [290, 41, 1]), ([9000], [70]), ([3000, 0], [33, 30])])
def test_attend_many_rows_of_any_group(dtype, Gq, lens, news):
    s = Step(lens, news, P=32, H=2, G=Gq, dtype=dtype, seed=Gq, spare=1)
    q = s.query(2.0)
    s.check(q, *s.attend(q), rows=sorted(set(list(range(0, s.real, 23)) + [s.real - 2, s.real - 1])))


@pytest.mark.parametrize("seed", range(24))
def test_attend_shares_of_units_of_any_length(seed):
    """Lengths, rows and masks by chance: units that are dealt out whole, in pieces and many to a workgroup, every few rows checked."""
    rng = np.random.default_rng(seed)
    B = int(rng.choice([1, 2, 5, 40]))
    top = {1: 40000, 2: 9000, 5: 5000, 40: 700}[B]
    lens = np.exp(rng.uniform(0, np.log(top), B)).astype(int).tolist()
    most = int(rng.choice([1, 2, 6, 40, 300])) if B < 40 else int(rng.choice([1, 3]))
    news = rng.integers(1, most + 1, B).tolist()
    s = Step(lens, news, P=int(rng.choice([16, 48, 128])), H=int(rng.choice([1, 3])), G=int(rng.choice([1, 4, 7])), seed=seed, dtype=["bf16", "f16"][seed % 2])
    q = s.query(2.0)
    kw = {}
    if seed % 3 == 1:
        kw["window"] = int(rng.integers(1, 2000))
    if seed % 3 == 2:
        kw["row_from"] = np.array([int(rng.integers(0, p + 2)) for p in s.pos], dtype=np.int32)      # no order among a sequence's rows
    if seed % 4 == 3:
        kw["prefix_len"] = rng.integers(0, top, B).astype(np.int32)
    s.check(q, *s.attend(q, **kw), rows=sorted(set(rng.integers(0, s.real, 24).tolist())), **kw)


def test_attend_many_short_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 60, 700).tolist()
    s = Step(lens, [1] * 700, H=2, G=2, seed=5)
    q = s.query()
    s.check(q, *s.attend(q), rows=range(0, 700, 9))
    s = Step(lens[:300], [2] * 300, H=2, G=2, seed=5)
    q = s.query()
    s.check(q, *s.attend(q), rows=range(0, 600, 11))


SCORES = [
    dict(softcap=30.0), dict(softcap=0.5), dict(softcap=1000.0), dict(slopes=True), dict(softcap=20.0, slopes=True), dict(window=1),
    dict(window=17), dict(window=300, softcap=30.0), dict(window=10 ** 9), dict(docs=50), dict(docs=1), dict(docs=333, window=100, slopes=True),
    dict(prefix=[100, 3, 10 ** 6]), dict(prefix=[-2 ** 31, 40, -5], window=30), dict(prefix=[2 ** 31 - 1] * 3, docs=90, slopes=True, softcap=9.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kw", SCORES, ids=str)
@pytest.mark.parametrize("lens,news,Gq", [([700, 0, 130], [1, 1, 1], 4), ([500, 2000, 0], [1, 1, 1], 7), ([300, 9, 0], [3, 1, 2], 5), ([0, 260, 31], [150, 40, 1], 4)])
def test_attend_with_scores_of_all_kinds(dtype, kw, lens, news, Gq):
    s = Step(lens, news, P=16 if Gq == 4 else 48, H=2, G=Gq, dtype=dtype, seed=len(kw))
    q = s.query(2.0)
    made = {n: kw[n] for n in ("softcap", "window") if n in kw}
    if "slopes" in kw:
        made["slopes"] = np.array([2.0 ** (-8 * (i + 1) / (2 * Gq)) * (-1 if i == 3 else 1) / (64 if i == 3 else 1) for i in range(2 * Gq)], dtype=np.float32)
    if "docs" in kw:
        made["row_from"] = np.array([p // kw["docs"] * kw["docs"] for p in s.pos], dtype=np.int32)
    if "prefix" in kw:
        made["prefix_len"] = np.array(kw["prefix"], dtype=np.int64).astype(np.int32)
    out, lse = s.attend(q, **made)
    s.check(q, out, lse, rows=range(0, s.real, 1 + s.real // 40), **made)


@pytest.mark.parametrize("softcap", [64.0, 65.0, 300.0, 3e4, 1e6, 2.0 ** 96])
@pytest.mark.parametrize("lens,news", [([700, 130], [1, 1]), ([300, 90], [9, 3]), ([200, 31], [90, 40])])
def test_large_caps(softcap, lens, news):
    """Logits of a few and of some hundreds, each as exact as without the cap however large that is."""
    for size in (1.0, 30.0):
        s = Step(lens, news, H=2, G=4, dtype="f16", seed=3)
        q = s.query(size)
        s.check(q, *s.attend(q, softcap=softcap), softcap=softcap, rows=range(0, s.real, 1 + s.real // 20))


@pytest.mark.parametrize("news", [[1, 1], [3, 2], [40, 7]])
def test_rows_that_see_nothing(news):
    s = Step([200, 60], news, H=2, G=3, seed=6)
    q = s.query()
    for first in ([p + 1 for p in s.pos], [2 ** 31 - 1] * s.T, [p + 1 if r % 2 else 0 for r, p in enumerate(s.pos)], [-2 ** 31] * s.T):
        row_from = np.array(first + [0] * (s.T - len(first)), dtype=np.int32)
        s.check(q, *s.attend(q, row_from=row_from), row_from=row_from)
    table = np.full_like(s.table, -1)                     # nothing is there
    s.rows.page_table.copy_(i32(table))
    s.check(q, *s.attend(q), table=table)


@pytest.mark.parametrize("news", [[1, 1], [9, 30]])
def test_attend_with_one_logit_far_above_the_rest_and_scales_far_apart(news):
    for dtype in ("bf16", "f16"):
        s = Step([700, 90], news, dtype=dtype, seed=8, exps=(-12, 3))
        q = s.query(6.0)
        s.check(q, *s.attend(q))


@pytest.mark.parametrize("lens,news", [([975], [2]), ([1000], [1]), ([973], [6]), ([965], [30])])
@pytest.mark.parametrize("gap", [14, 30, 80])
def test_a_page_of_large_values_costs_rows_that_do_not_see_it_nothing(lens, news, gap):
    s = Step(lens, news, H=1, seed=gap)
    last = int(s.table[0, (lens[0] + news[0] - 1) // 16])
    s.cache.pages[last, :, :, 2112:] = 127 + 10
    s.cache.pages[s.table[0, 0], :, :, 2112:] = 127 + 10 - gap
    first = s.pos[0] // 16 * 16
    behind = [r for r, p in enumerate(s.pos) if p // 16 < (lens[0] + news[0] - 1) // 16]
    q = s.query(0.5)
    hide = np.array([min(p, first) if news[0] == 1 else 0 for p in s.pos], dtype=np.int32) * 0
    out, lse = s.attend(q, row_from=hide)
    s.check(q, out, lse, row_from=hide)
    if behind:
        s.cache.pages[last, :, :, 2112:] = 127
        again, _ = s.attend(q, row_from=hide)
        assert torch.equal(again[behind], out[behind])


def test_values_at_the_top_of_the_range_are_numbers():
    """bf16: magnitudes of up to 6 * 2^125, and their averages."""
    for lens, news in (([1000], [1]), ([500], [6]), ([300], [40])):
        s = Step(lens, news, H=2, seed=41)
        s.cache.pages[..., 2112:] = 127 + 125
        q = s.query(0.5)
        s.check(q, *s.attend(q))


def test_small_values_and_keys():
    for lens, news in (([1000], [1]), ([300], [40])):
        s = Step(lens, news, H=2, seed=42)
        s.cache.pages[..., 2112:] = 127 - 60
        s.cache.pages[..., 2048:2112] = 127 - 80
        q = s.query(0.5)
        s.check(q, *s.attend(q))


def test_attend_strided_queries_no_lse_and_a_scale_of_its_own():
    s = Step([50, 90], [3, 1], seed=9)
    wide = s.randn(s.T, s.H * s.G + 4, D)
    q = wide[:, 1:1 + s.H * s.G]
    out, lse = s.attend(q)
    s.check(q, out, lse)
    again, none = s.attend(q, lse=False)
    assert none is None and torch.equal(again, out)
    s = Step([50, 90], [3, 1], seed=9, scale=0.31)
    q = s.query()
    s.check(q, *s.attend(q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_queries_far_apart_in_size(dtype):
    s = Step([300, 40], [5, 6], dtype=dtype, seed=19)
    q = s.query()
    q[0] *= 2.0 ** -9
    q[1, :, 7] *= 300.0
    q[2] = 0.0
    q[3, 1] = 2.0 ** -14
    s.check(q, *s.attend(q))


@pytest.mark.parametrize("news", [[1, 1, 1], [5, 2, 20]])
def test_attend_keeps_bad_blocks_and_hidden_tokens_out(news):
    s = Step([300, 40, 0], news, seed=10)
    table = s.table.copy()
    table[0, 2], table[0, 5], table[2, 0] = -1, s.NB, -2 ** 31
    s.rows.page_table.copy_(i32(table))
    q = s.query()
    s.check(q, *s.attend(q), table=table)
    # what lies behind a sequence's last token, and in pages that nobody reads, has no influence: scales that are infinite or no number
    before = s.attend(q)
    _, _, ks, vs = R.places(16)
    end = 300 + news[0]
    flat = s.cache.pages.view(s.NB, s.H, -1)
    last = int(table[0, (end - 1) // 16])
    for t in range(end % 16, 16) if end % 16 else ():
        for at in (ks[t], vs[t]):
            flat[last][:, torch.from_numpy(at).to(DEV)] = 255
    used = set(table[(table >= 0) & (table < s.NB)].tolist())
    for b in set(range(s.NB)) - used:
        s.cache.pages[b] = 255
    after = s.attend(q)
    assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [5, 6, 1, 1], [40, 6, 0, 0]])
def test_a_row_that_is_no_number_stays_alone(bad, news):
    s = Step([300, 40, 5, 700], news, seed=11)
    q = s.query()
    good, glse = s.attend(q)
    q2 = q.clone()
    q2[3, 2, 7] = bad
    out, lse = s.attend(q2)
    assert torch.isnan(out[3, 2]).all() and torch.isnan(lse[3, 2])
    out[3, 2], lse[3, 2] = good[3, 2], glse[3, 2]
    assert torch.equal(out, good) and torch.equal(lse, glse)


# ---- streams, graphs, workspaces, the whole ----------------------------------------------------------

def test_calls_on_two_streams_with_a_workspace_each():
    a, b = Step([9000, 40], [1, 1], seed=13), Step([5000, 700, 3], [7, 1, 2], dtype="f16", seed=14)
    qa, qb = a.query(), b.query()
    wa, wb = a.attend(qa), b.attend(qb, softcap=20.0)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    wsa, wsb = a.cache.workspace(a.rows), b.cache.workspace(b.rows)
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        with torch.cuda.stream(sa):
            got.append((a.attend(qa, ws=wsa), wa))
        with torch.cuda.stream(sb):
            got.append((b.attend(qb, ws=wsb, softcap=20.0), wb))
    torch.cuda.synchronize()
    for (o, l), (wo, wl) in got:
        assert torch.equal(o, wo) and torch.equal(l, wl)
    # every call leaves the workspace ready: the counters at its start are zero again
    assert int(wsa[:2048].abs().max()) == 0 and int(wsb[:2048].abs().max()) == 0


def test_results_do_not_change_from_call_to_call():
    s = Step([40000, 0, 1234, 3], [1, 1, 1, 1], H=2, G=5, seed=15)
    q = s.query()
    first = s.attend(q)
    for _ in range(20):
        o, l = s.attend(q)
        assert torch.equal(o, first[0]) and torch.equal(l, first[1])


def test_one_workspace_for_calls_of_different_sizes():
    steps = [Step([9000, 40], [1, 1], seed=21), Step([600, 700], [40, 9], dtype="f16", seed=22), Step([5000], [3], P=32, G=8, seed=23)]
    ws = torch.zeros(max(s.cache.workspace(s.rows).numel() for s in steps), dtype=torch.int32, device=DEV)
    qs = [s.query() for s in steps]
    alone = [s.attend(q) for s, q in zip(steps, qs)]
    for _ in range(3):
        for s, q, want in zip(steps, qs, alone):
            out, lse = s.attend(q, ws=ws)
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert int(ws[:2048].abs().max()) == 0


class Server:
    """A serving loop: requests of growing length, their pages and blocks, one layer."""

    def __init__(self, B, NP, NB, T, P=16, H=2, Gq=4, dtype="bf16"):
        self.P, self.H, self.G, self.NB = P, H, Gq, NB
        self.dt = torch_type(dtype)
        self.cache = K.Q4Cache(n_blocks=NB, n_q_heads=H * Gq, n_kv_heads=H, page_size=P, kv_dtype=self.dt, device=DEV)
        self.rows = K.Q8Rows(torch.full((B, NP), -1, dtype=torch.int32, device=DEV), page_size=P, n_blocks=NB, n_rows=T)
        self.freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float()
        g = torch.Generator(device=DEV)
        g.manual_seed(77)
        self.wq, self.wk = ((1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(self.dt) for _ in range(2))
        self.rotary = K.Rotary(self.freq.to(DEV), n_q_heads=H * Gq, n_kv_heads=H, kv_dtype=self.dt, q_weight=self.wq, k_weight=self.wk)
        self.seq_len, self.n_new = i32([0] * B), i32([0] * B)
        self.free = i32(np.random.default_rng(0).permutation(NB))
        self.count = i32([NB])
        self.qkv = torch.zeros((T, H * Gq + 2 * H, D), dtype=self.dt, device=DEV)
        self.q, self.kn = (torch.zeros((T, n, D), dtype=self.dt, device=DEV) for n in (H * Gq, H))
        self.out = torch.zeros_like(self.q)
        self.kb, self.vb = torch.zeros_like(self.kn), torch.zeros_like(self.kn)
        self.lse = torch.zeros((T, H * Gq), device=DEV)
        self.ws = self.cache.workspace(self.rows)

    def step(self):
        n, H = self.H * self.G, self.H
        self.rows.map(self.seq_len, self.n_new, self.free, self.count)
        self.rotary.apply(self.rows.row_pos, self.qkv[:, :n], self.qkv[:, n:n + H], q_out=self.q, k_out=self.kn)
        self.cache.append(self.rows, self.kn, self.qkv[:, n + H:])
        self.cache.attend(self.rows, self.q, self.out, self.ws, lse=self.lse, softcap=50.0, window=100)
        self.cache.read(self.rows, self.kb, self.vb)
        self.seq_len.copy_(self.rows.kv_len)
        self.count.copy_(self.rows.counts[3:4])

    def results(self):
        return [t.clone() for t in (self.q, self.kn, self.out, self.lse, self.kb, self.vb, self.cache.pages, self.rows.page_table, self.rows.kv_len,
                                    self.count)]


def _feed(server, i, news):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000 + i)
    server.qkv.copy_(torch.randn(server.qkv.shape, generator=g, device=DEV))
    server.n_new.copy_(i32(news))


def test_serving_steps_together():
    """Prompts, then single tokens, then drafts with some requests resting: every step against the definition."""
    B, NP, NB, T, P = 3, 30, 80, 150, 16
    s = Server(B, NP, NB, T)
    table, ref = np.full((B, NP), -1), R.Cache(NB, s.H, P)
    lens, count, free = [0] * B, NB, s.free.cpu().tolist()
    for i, news in enumerate([[100, 0, 37], [1, 1, 1], [1, 9, 1], [0, 3, 2], [60, 1, 60], [1, 1, 1], [2, 0, 2]]):
        _feed(s, i, news)
        s.step()
        want = R8.map_step(lens, news, table, free, count, P, T, s.rows.max_runs)
        lens, count = want["kv_len"], want["counts"][3]
        n, rows = s.H * s.G, want["counts"][0]
        x, pos = s.qkv.double().cpu().numpy(), [want["row_pos"][:rows]]
        for got, y, w in ((s.q, x[:rows, :n], s.wq), (s.kn, x[:rows, n:n + s.H], s.wk)):
            y, size = R.rotate(y, pos, s.freq.double().numpy(), weight=w.double().cpu().numpy())
            assert (np.abs(got[:rows].double().cpu().numpy() - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * size).all()
        ref.append(want["runs"], s.kn.double().cpu().numpy(), x[:, n + s.H:])
        assert np.array_equal(s.rows.page_table.cpu().numpy(), table) and s.rows.counts.cpu().tolist() == want["counts"]
        got = R.Cache.of_bytes(s.cache.pages.cpu().numpy(), P)
        used = sorted(set(table[table >= 0].tolist()))
        assert np.array_equal(got.codes[used], ref.codes[used]) and np.array_equal(got.exps[used], ref.exps[used])
        q = s.q.double().cpu().numpy()
        for r in range(0, rows, 5):
            b, p = want["row_seq"][r], want["row_pos"][r]
            for h in range(s.H):
                at = R.Row(ref, table[b], q[r, h * s.G:(h + 1) * s.G], h, p, max(0, p - 99), p, 1.0 / np.sqrt(128.0), 50.0)
                g = s.out[r, h * s.G:(h + 1) * s.G].double().cpu().numpy()
                # half a step of bf16 each for the output and for the weights, 2^-12 for all else, with |v| below 6 in any average
                assert np.abs(g - at.out).max() <= 2.0 ** -8 * np.abs(at.out).max() + (2.0 ** -8 + 2.0 ** -12) * 6.0, (i, r, h)
                t = p % P
                kv = [R.number(ref.codes[table[b][p // P], h, w, t], np.repeat(ref.exps[table[b][p // P], h, w, t], 32)) for w in (0, 1)]
                assert np.array_equal(s.kb[r, h].double().cpu().numpy(), kv[0]) and np.array_equal(s.vb[r, h].double().cpu().numpy(), kv[1])


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
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
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
