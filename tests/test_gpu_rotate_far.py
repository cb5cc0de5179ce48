"""Angles of far positions: up to 2^29 turns, of which the fraction has to be right to 2^-24."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd as K
from tests.q8_rig import DEV, D, i32

pytestmark = pytest.mark.gpu

PER_RADIAN = Fraction("0.159154943091895335768883763372514362034459645740456448747667")      # 1 / (2 pi)
# frequencies whose turns come out far off in 53 bits, and positions of theirs that are nearly whole turns, whose sines show it
FREQ = [1.5729098320007324, 1.5779577493667603, 1.0, 0.8969]
POS = [2144566116, 2144579494, 2144592872, 2137698042, 2137716028, 2137734014, 2141034100, 2 ** 31 - 1, -2144566116, -2137698042, -2 ** 31]


def _fraction(pos, f):
    turns = pos * Fraction(f) * PER_RADIAN
    return float(turns - round(turns))


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("T", [len(POS), 2100])
def test_fractions_of_many_turns(near, T):
    n = 64
    f = torch.tensor([FREQ[i % 4] for i in range(n)], dtype=torch.float32)
    pos = [POS[i % len(POS)] for i in range(T)]
    a = torch.zeros((T, 2, D), dtype=torch.float16, device=DEV)
    first, second = (slice(0, None, 2), slice(1, None, 2)) if near else (slice(0, n), slice(n, None))
    a[:, 0, first] = 1024.0                                  # the first head has (1024, 0), the other one (0, 1024)
    a[:, 1, second] = 1024.0
    r = K.Rotary(f.to(DEV), n_q_heads=2, n_kv_heads=1, kv_dtype=torch.float16, interleaved=near, axis_pairs=[0, n])
    out = torch.empty_like(a)
    r.apply(i32([[0] * T, pos]), a, q_out=out)               # (axis 0 has to be a row's position; the other one may be below zero)
    got = out[: len(POS)].double().cpu().numpy()
    turn = np.array([[_fraction(p, float(x)) for x in f[:4]] for p in POS])
    cos, sin = (np.tile(1024 * g(2 * math.pi * turn), (1, n // 4)) for g in (np.cos, np.sin))
    for h, (one, two) in enumerate(((cos, sin), (-sin, cos))):
        for x, want in ((got[:, h, first], one), (got[:, h, second], two)):
            # half a step of f16, and 2^-24 of a turn
            bad = ~(np.abs(x - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + 1024 * 2 * math.pi * 2.0 ** -24)
            assert not bad.any(), (h, np.argwhere(bad)[:4].tolist(), np.abs(x - want).max())
    assert all(torch.equal(out[i:i + len(POS)], out[: len(POS)]) for i in range(0, T - len(POS), len(POS)))
