"""How exactly the 4-bit cache's attention weighs values: small logits and few tokens, whose values cancel in the average, so that a
weight's own rounding is what an output is off by.  One case for each layout of the query rows and each kind of scores."""
import math

import numpy as np
import pytest
import torch

from tests import q4_ref as R
from tests.q4_rig import D, Step

pytestmark = pytest.mark.gpu

# average columns of a sequence (rows times heads of the group): 4, 8, 16, 32, 64, 128, 256
FORMS = [([5, 2, 40], [1, 1, 1], 4), ([3, 9], [2, 2], 4), ([4, 30, 1], [4, 4, 4], 4), ([2, 17], [8, 8], 4), ([6, 300], [16, 16], 4),
         ([0, 5], [32, 32], 4), ([1, 60], [64, 64], 4)]
SCORES = [{}, dict(softcap=20.0), dict(softcap=500.0), dict(slopes=True), dict(window=5)]


def _bound(x, dtype, softcap):
    """An output is off by at most half a step of its type, by the two parts of a weight, 2^-16 of it, by twice the logits' error (128 products
    in fp32, 2^-17 of their sum; a cap's 2^-20 of it, or of the logit above 64; a bias's 2^-22; the exponent's argument, 2^-23 of it,
    and 2^-20), by the sums' and joins' 2^-17 and by half of f16's least step."""
    dx = 2.0 ** -17 * x.products + 2.0 ** -20 * (1 + (softcap if softcap <= 64 else x.capped)) + 2.0 ** -22 * x.bias + 2.0 ** -23 * x.largest
    tol = torch.finfo(dtype).eps / 2 * np.abs(x.out) + (2.0 ** -16 + 2.0 ** -17 + 2 * dx[:, None]) * x.mass
    return tol + (2.0 ** -25 if dtype == torch.float16 else 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kw", SCORES, ids=str)
@pytest.mark.parametrize("lens,news,Gq", FORMS)
def test_weights_have_sixteen_bits(dtype, kw, lens, news, Gq):
    s = Step(lens, news, H=2, G=Gq, dtype=dtype, seed=len(lens) + Gq)
    q = s.query(0.05)
    made = dict(kw)
    if "slopes" in kw:
        made["slopes"] = np.array([2.0 ** -(2 + i) for i in range(2 * Gq)], dtype=np.float32)
    out, _ = s.attend(q, **made)
    ref, qd, od = s.ref(), q.double().cpu().numpy(), out.double().cpu().numpy()
    for row in range(0, s.real, 1 + s.real // 48):
        pos = s.pos[row]
        lo = max(0, pos - kw["window"] + 1) if "window" in kw else 0
        for h in range(2):
            heads = slice(h * Gq, (h + 1) * Gq)
            x = R.Row(ref, s.table[s.seq[row]], qd[row, heads], h, pos, lo, pos, 1.0 / math.sqrt(D), kw.get("softcap", 0.0),
                      made["slopes"][heads].astype(np.float64) if "slopes" in kw else None)
            off, bound = np.abs(od[row, heads] - x.out), _bound(x, out.dtype, kw.get("softcap", 0.0))
            bad = ~(off <= bound)
            assert not bad.any(), f"row {row} head {h}: {(off[bad] / bound[bad]).max()} times the bound, {bad.sum()} of {bad.size}"
