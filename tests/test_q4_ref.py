"""The 64-bit definition of the 4-bit cache (tests/q4_ref.py) against values worked by hand.  No GPU needed."""
import math

import numpy as np
import pytest

from tests import q4_ref as R


def test_numbers_and_roundings():
    assert R.number([0, 1, 2, 3, 4, 5, 6, 7, 9, 15], [0] * 10).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -6]
    x = np.zeros(128)
    x[:12] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -6.5, 0.2500001, 5.0000001]
    code, e = R.quantise(x)
    assert e.tolist() == [0, -96, -96, -96]
    assert code[:12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 15, 1, 7]


@pytest.mark.parametrize("amax,e", [(7.0, 0), (7.0000001, 1), (3.5, -1), (1.0, -2), (0.0, -96), (2.0 ** -99, -96), (7 * 2.0 ** 125, 125), (2.0 ** 128, 125), (65504.0, 14)])
def test_exponents(amax, e):
    assert R.exponent(amax) == e


def test_what_is_no_number():
    x = np.ones(128)
    x[0], x[1], x[2], x[40], x[3] = math.inf, -math.inf, math.nan, math.inf, -0.0
    code, e = R.quantise(x)
    assert e.tolist() == [-2, -2, -2, -2] and code[[0, 1, 2, 3, 4, 40]].tolist() == [7, 15, 0, 8, 6, 7]


def test_places_are_a_permutation_and_bytes_come_back():
    for P in (16, 48):
        key, val, ks, vs = R.places(P)
        codes = np.concatenate([key.flatten(), val.flatten()])
        assert len(set(codes.tolist())) == 2 * P * 128
        used = set((codes // 2).tolist()) | set(ks.flatten().tolist()) | set(vs.flatten().tolist())
        assert used == set(range(P // 16 * 2176))
        raw = np.random.default_rng(P).integers(0, 256, (3, 2, P // 16, 2176)).astype(np.uint8)
        assert np.array_equal(R.Cache.of_bytes(raw, P).bytes(), raw)


def test_attention_of_two_tokens_by_hand():
    c = R.Cache(1, 1, 16)
    k, v = np.zeros((2, 1, 128)), np.zeros((2, 1, 128))
    k[1, 0, 0], v[0, 0, 0], v[1, 0, 0] = 1.0, 1.0, 4.0
    c.append([[0, 0, 0, 2]], k, v)
    x = np.zeros((1, 128))
    x[0, 0] = math.log(3.0)
    r = R.Row(c, np.array([0]), x, 0, 1, 0, 1, 1.0)
    assert math.isclose(r.out[0, 0], (1 + 3 * 4) / 4) and math.isclose(r.lse[0], math.log(4.0)) and math.isclose(r.mass[0, 0], 3.25)
    r = R.Row(c, np.array([0]), x, 0, 1, 0, 1, 1.0, slopes=np.array([math.log(3.0)]))
    assert math.isclose(r.out[0, 0], (1 / 3 + 3 * 4) / (3 + 1 / 3))
    r = R.Row(c, np.array([0]), x, 0, 1, 0, 1, 1.0, cap=0.5)
    assert math.isclose(r.lse[0], math.log(1 + math.exp(0.5 * math.tanh(2 * math.log(3.0)))))
    assert R.Row(c, np.array([0]), x, 0, 1, 2, 1, 1.0).empty and R.Row(c, np.array([-1]), x, 0, 1, 0, 1, 1.0).empty


def test_a_quarter_turn():
    x = np.arange(128.0).reshape(1, 1, 128)
    f = np.array([math.pi / 2] + [0.0] * 7)
    y, _ = R.rotate(x, [[1]], f)
    assert np.allclose(y[0, 0, [0, 8]], [-8, 0]) and np.array_equal(y[0, 0, 16:], x[0, 0, 16:]) and y[0, 0, 1] == 1
    y, _ = R.rotate(x, [[1], [3]], f, interleaved=True, axis_pairs=[0, 8])
    assert np.allclose(y[0, 0, :2], [1, 0])                   # three quarter turns of (0, 1)
    y, _ = R.rotate(x[:, :, :], [[5]], [], weight=np.full(128, 2.0), eps=0.0)
    assert math.isclose((y ** 2).mean(), 4.0)
