"""The serving loop that README.md shows, run as it stands there."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd
from tests import q8_ref as R
from tests.q8_rig import DEV, D, i32

pytestmark = pytest.mark.gpu


def test_the_loop_of_the_readme():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    loop = next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "Q8Cache" in b)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    new = lambda h: torch.randn((64, h, D), generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    plan = [[30, 5, 0], [1, 1, 1], [2, 0, 40], [1, 1, 1]]
    steps = [(i32(n), new(32), new(8), new(8)) for n in plan]
    names = dict(torch=torch, kvd=kvd, steps=steps, page_table=i32(np.full((3, 12), -1)), seq_len=i32([0, 0, 0]),
                 free_blocks=i32(np.random.default_rng(0).permutation(4096)), free_count=i32([4096]), out=torch.zeros_like(steps[0][1]),
                 lse=torch.zeros((64, 32), device=DEV))
    free = names["free_blocks"].tolist()
    exec(loop, names)
    lens, count, table, ref = [0, 0, 0], 4096, np.full((3, 12), -1), R.Cache(4096, 8, 16)
    for (_, q, k, v), n in zip(steps, plan):
        want = R.map_step(lens, n, table, free, count, 16, 64, names["rows"].max_runs)
        lens, count = want["kv_len"], want["counts"][3]
        ref.append(want["runs"], k.double().cpu().numpy(), v.double().cpu().numpy())
    assert names["seq_len"].tolist() == lens == [34, 7, 42] and names["free_count"].tolist() == [count]
    assert np.array_equal(names["page_table"].cpu().numpy(), table)
    assert np.array_equal(names["cache"].pages.cpu().numpy(), ref.bytes())
    for r in range(3):
        for h in range(0, 8, 3):
            x = steps[-1][1][r, 4 * h:4 * h + 4].double().cpu().numpy()
            o, _ = R.attend_row(ref, table[r], x, h, lens[r] - 1, 1.0 / np.sqrt(128.0))
            # half a step of bf16 each for the output and for P, with |v| below 5 in any average
            assert np.abs(names["out"][r, 4 * h:4 * h + 4].double().cpu().numpy() - o).max() <= 2.0 ** -8 * (np.abs(o).max() + 5.0), (r, h)
