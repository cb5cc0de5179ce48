"""The plain definition of the 8-bit paged cache against things that are known without it.  No GPU needed."""
import numpy as np
import torch

from tests import q8_ref as R


def test_codes_are_those_of_torch_and_round_to_even():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.VALUES, want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20011), np.linspace(-0.05, 0.05, 4001),
                        (R._POS[:-1] + R._POS[1:]) / 2, -(R._POS[:-1] + R._POS[1:]) / 2]).astype(np.float32)
    got = R.encode(x.astype(np.float64))
    assert np.array_equal(got, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_exponent_is_the_least_that_holds_the_largest():
    for top in (448.0, 448.0000001, 447.0, 1.0, 0.875, 1.75, 1.7500001, 3e38, 1e-20, 6e-8):
        e = R.exp_for(np.array([top, -top / 3, np.nan, np.inf]))
        assert top <= 448.0 * 2.0 ** e and top > 448.0 * 2.0 ** (e - 1)
    assert R.exp_for(np.array([0.0, np.nan])) == R.EXP_MIN and R.exp_for(np.array([1e-40])) == R.EXP_MIN


def test_places_of_a_page_are_all_different():
    for P in (16, 48, 256):
        key, val = R.tile_places(P)
        at = np.concatenate([key.ravel(), val.ravel()])
        assert np.array_equal(np.sort(at), np.arange(P * 256))


def test_append_in_pieces_keeps_the_scale_rule():
    rng = np.random.default_rng(0)
    c = R.Cache(2, 1, 32)
    k = rng.standard_normal((32, 1, 128))
    k[20:] *= 40.0
    c.append([[1, 0, 0, 20]], k, k)
    e0 = c.exps[1, 0, 0]
    first = c.kv([1], 0)[0][:20]
    assert np.abs(first - k[:20, 0]).max() <= 2.0 ** -4 * np.abs(k[:20]).max()
    c.append([[1, 20, 20, 12]], k, k)
    assert c.exps[1, 0, 0] > e0
    got = c.kv([1], 0)[0]
    # a value is off by half a step of 2^-4 of itself at most, twice where the scale grew, or by half the smallest step
    assert (np.abs(got - k[:, 0]) <= 0.13 * np.abs(k[:, 0]) + 2.0 ** (c.exps[1, 0, 0] - 9)).all()
    mean = c.means[1, 0] * float(c.mean_scales[1, 0])
    assert np.abs(mean - got.mean(0)).max() <= np.abs(got.mean(0)).max() / 120


def test_map_rows_runs_and_blocks_by_hand():
    table = np.full((3, 4), -1)
    table[0, 0] = 9
    got = R.map_step([10, 0, 0], [8, 0, 33], table, [5, 6, 7, 8], 4, 16, 48, 9)
    assert got["counts"] == [41, 5, 4, 0, 0]
    assert table.tolist() == [[9, 8, -1, -1], [-1] * 4, [7, 6, 5, -1]]
    assert got["runs"][:5] == [[9, 0, 10, 6], [8, 6, 0, 2], [7, 8, 0, 16], [6, 24, 0, 16], [5, 40, 0, 1]]
    assert got["row_start"] == [0, 8, 8, 41] and got["kv_len"] == [18, 0, 33]
    assert got["row_pos"][:9] == [10, 11, 12, 13, 14, 15, 16, 17, 0] and got["row_seq"][40:43] == [2, -1, -1]
    before = table.copy()
    assert R.map_step([18, 0, 33], [0, 1, 0], table, [5, 6, 7, 8], 0, 16, 48, 9)["counts"] == [0, 0, 0, 0, 1]
    assert np.array_equal(before, table)


def test_attention_of_equal_keys_is_the_mean_of_the_values():
    c = R.Cache(3, 1, 16)
    k = np.ones((40, 1, 128))
    v = np.random.default_rng(1).standard_normal((40, 1, 128))
    c.append([[2, 0, 0, 16], [0, 16, 0, 16], [1, 32, 0, 8]], k, v)
    out, lse = R.attend_row(c, [2, 0, 1], np.ones((2, 128)), 0, 39, 0.5)
    vals = np.concatenate([c.kv([b], 0)[1] for b in (2, 0, 1)])[:40]
    assert np.allclose(out, vals.mean(0)) and np.allclose(lse, np.log(40) + 64.0)
    assert R.attend_row(c, [-1, 0, 1], np.ones((1, 128)), 0, 3, 0.5)[1][0] == -np.inf
