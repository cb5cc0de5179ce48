"""The serving loop of the 4-bit cache that README.md shows, run as it stands there."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd
from tests import q4_ref as R
from tests import q8_ref as R8
from tests.q8_rig import DEV, D, i32

pytestmark = pytest.mark.gpu


def test_the_loop_of_the_readme():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    loop = next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "Q4Cache" in b)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    new = lambda h: torch.randn((64, h, D), generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    plan = [[30, 5, 0], [1, 1, 1], [2, 0, 40], [1, 1, 1]]
    steps = [(i32(n), new(32), new(8), new(8)) for n in plan]
    before = [(q.clone(), k.clone()) for _, q, k, _ in steps]
    names = dict(torch=torch, kvd=kvd, steps=steps, page_table=i32(np.full((3, 12), -1)), seq_len=i32([0, 0, 0]),
                 free_blocks=i32(np.random.default_rng(0).permutation(4096)), free_count=i32([4096]), out=torch.zeros_like(steps[0][1]),
                 lse=torch.zeros((64, 32), device=DEV), inv_freq=(10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().to(DEV),
                 q_weight=1 + 0.1 * new(1)[0, 0], k_weight=1 + 0.1 * new(1)[0, 0], k_held=new(8), v_held=new(8))
    free = names["free_blocks"].tolist()
    exec(loop, names)
    lens, count, table, ref = [0, 0, 0], 4096, np.full((3, 12), -1), R.Cache(4096, 8, 16)
    freq = names["inv_freq"].double().cpu().numpy()
    for (_, q, k, v), (q0, k0), n in zip(steps, before, plan):
        want = R8.map_step(lens, n, table, free, count, 16, 64, names["rows"].max_runs)
        lens, count, real = want["kv_len"], want["counts"][3], want["counts"][0]
        for got, x, w in ((q, q0, "q_weight"), (k, k0, "k_weight")):
            y, size = R.rotate(x[:real].double().cpu().numpy(), [want["row_pos"][:real]], freq, weight=names[w].double().cpu().numpy())
            assert (np.abs(got[:real].double().cpu().numpy() - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * size).all()
            assert torch.equal(got[real:], x[real:])
        ref.append(want["runs"], k.double().cpu().numpy(), v.double().cpu().numpy())
    assert names["seq_len"].tolist() == lens == [34, 7, 42] and names["free_count"].tolist() == [count]
    assert np.array_equal(names["page_table"].cpu().numpy(), table)
    got = R.Cache.of_bytes(names["cache"].pages.cpu().numpy(), 16)
    used = sorted(set(table[table >= 0].tolist()))
    assert np.array_equal(got.codes[used], ref.codes[used]) and np.array_equal(got.exps[used], ref.exps[used])
    for r in range(3):
        t, block = (lens[r] - 1) % 16, table[r][(lens[r] - 1) // 16]
        for h in range(0, 8, 3):
            x = steps[-1][1][r, 4 * h:4 * h + 4].double().cpu().numpy()
            at = R.Row(ref, table[r], x, h, lens[r] - 1, 0, lens[r] - 1, 1.0 / np.sqrt(128.0), 50.0)
            # half a step of bf16 each for the output and for the weights, 2^-12 for all else, with |v| below 6 in any average
            assert np.abs(names["out"][r, 4 * h:4 * h + 4].double().cpu().numpy() - at.out).max() <= 2.0 ** -8 * np.abs(at.out).max() + (2.0 ** -8 + 2.0 ** -12) * 6.0
            for which, held in ((0, names["k_held"]), (1, names["v_held"])):
                assert np.array_equal(held[r, h].double().cpu().numpy(), R.number(ref.codes[block, h, which, t], np.repeat(ref.exps[block, h, which, t], 32)))
