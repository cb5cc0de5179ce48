"""Norm and rotation of query and key heads on the GPU against their 64-bit definition (tests/q4_ref.py)."""
import numpy as np
import pytest
import torch

from paper_2605_18071_amd import kvd as K
from tests import q4_ref as R
from tests.q8_rig import DEV, D, i32, torch_type

pytestmark = pytest.mark.gpu


def _check(got, x, size, dtype):
    """An element is off by at most half a step of its type, 2^-18 of what its pair is made of (128 squares and their sum in fp32, a
    root, a product: 2^-20; a sine to 2^-21), and half of f16's least step."""
    tol = torch.finfo(torch_type(dtype)).eps / 2 * np.abs(x) + 2.0 ** -18 * size + (2.0 ** -25 if dtype == "f16" else 0.0)
    bad = ~(np.abs(got - x) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), np.abs(got - x)[bad].max(), tol[bad].min())


def _freq(n, base=10000.0):
    return (base ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))).float()


def _run(T, Hq, Hk, dtype, rot, near, pairs, norm, pos, seed, *, in_place=False, base=10000.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch_type(dtype)
    wide = (torch.randn((T, Hq + 2 * Hk + 1, D), generator=g, device=DEV) * 3).to(dt)
    q, k = wide[:, :Hq], wide[:, Hq:Hq + Hk]
    wq, wk = ((1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) for _ in range(2))
    wq, wk = wq if norm & 1 else None, wk if norm & 2 else None
    f = _freq(rot // 2, base)
    r = K.Rotary(f.to(DEV), n_q_heads=Hq, n_kv_heads=Hk, kv_dtype=dt, interleaved=near, axis_pairs=pairs, q_weight=wq, k_weight=wk, eps=1e-5)
    x = [t.double().cpu().numpy() for t in (q, k)]
    rest = wide[:, Hq + Hk:].clone()
    outs = (q, k) if in_place else [torch.full(t.shape, 7.0, dtype=dt, device=DEV) for t in (q, k)]
    p = i32(pos)
    r.apply(p, q, k, **({} if in_place else dict(q_out=outs[0], k_out=outs[1])))
    real = np.asarray(pos).reshape(-1, T)[0] >= 0
    for got, y, w in zip(outs, x, (wq, wk)):
        want, size = R.rotate(y[real], np.asarray(pos).reshape(-1, T)[:, real], f.double().numpy(), interleaved=near, axis_pairs=pairs,
                              weight=None if w is None else w.double().cpu().numpy(), eps=1e-5)
        got = got.double().cpu().numpy()
        _check(got[real], want, size, dtype)
        assert (got[~real] == (y[~real] if in_place else 7.0)).all()
    assert torch.equal(wide[:, Hq + Hk:], rest)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 96, 128])
@pytest.mark.parametrize("T,Hq,Hk", [(1, 1, 1), (3, 7, 1), (130, 32, 8), (2050, 5, 2)])
def test_rotate(dtype, near, rot, T, Hq, Hk):
    pos = np.random.default_rng(T).integers(0, 200000, T)
    _run(T, Hq, Hk, dtype, rot, near, None, 3, pos, T + rot)


@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("near", [False, True])
def test_rotate_with_and_without_norms_in_place_and_out(norm, near):
    pos = np.arange(37)
    _run(37, 6, 3, "bf16", 128, near, None, norm, pos, 1)
    _run(37, 6, 3, "f16", 96, near, None, norm, pos, 2, in_place=True)
    _run(3000, 6, 3, "bf16", 64, near, None, norm, np.arange(3000), 3, in_place=True)


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("pairs", [[16, 24, 24], [0, 64], [20, 20, 4, 20], [64]])
def test_several_axes(near, pairs):
    rng = np.random.default_rng(5)
    for T in (19, 2100):
        _run(T, 4, 2, "bf16", 128, near, pairs, 3, rng.integers(0, 5000, (len(pairs), T)), 4)


def test_negative_positions_of_other_axes_turn_back():
    pos = np.array([[0, 5, 9], [-3, 0, -2 ** 31], [7, -7, 2 ** 31 - 1]])
    _run(3, 2, 2, "f16", 96, False, [8, 20, 20], 3, pos, 6)


@pytest.mark.parametrize("base", [10000.0, 5e6, 1.0])
def test_far_positions(base):
    """Frequencies of 1 at positions up to 2^31: more turns than fp32 could hold the fraction of."""
    _run(6, 2, 1, "f16", 128, False, None, 0, [0, 1, 2 ** 20 + 1, 2 ** 24 + 1, 2 ** 30 - 3, 2 ** 31 - 1], 7, base=base)


@pytest.mark.parametrize("T", [9, 2060])
def test_rows_without_a_token_are_left_out(T):
    pos = np.arange(T)
    pos[[0, 3, 4]] = -1
    pos[T - 3:] = -1
    _run(T, 32, 8, "bf16", 128, False, None, 3, pos, 8)
    _run(T, 3, 1, "bf16", 128, True, None, 3, pos, 8, in_place=True)


def test_one_of_the_two_alone():
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    q, k = (torch.randn((50, h, D), generator=g, device=DEV).half() for h in (9, 4))
    pos = i32(np.arange(50))
    r = K.Rotary(_freq(64).to(DEV), n_q_heads=9, n_kv_heads=4, kv_dtype=torch.float16)
    both = torch.empty_like(q), torch.empty_like(k)
    r.apply(pos, q, k, q_out=both[0], k_out=both[1])
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    r.apply(pos, q, q_out=q2)
    r.apply(pos, None, k, k_out=k2)
    assert torch.equal(q2, both[0]) and torch.equal(k2, both[1])


def test_numbers_at_the_ends_of_the_range_and_none():
    q = torch.zeros((4, 2, D), dtype=torch.bfloat16, device=DEV)
    q[1, 0] = 2.0 ** -70                                     # squares far below eps
    q[2, 1] = 2.0 ** 58                                      # a sum of squares of 2^123
    q[3, 0, 5] = float("nan")
    q[3, 1] = 1.0
    w = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    r = K.Rotary(_freq(0).to(DEV), n_q_heads=2, n_kv_heads=1, kv_dtype=torch.bfloat16, q_weight=w, eps=1e-6)
    out = torch.empty_like(q)
    r.apply(i32([0, 1, 2, 3]), q, q_out=out)
    assert (out[0] == 0).all() and (out[2, 1] == 1).all() and (out[3, 1] == 1).all() and torch.isnan(out[3, 0]).all()
    assert ((out[1, 0].double() - 1000 * 2.0 ** -70).abs() <= 1000 * 2.0 ** -78).all()


def test_rotation_in_a_graph():
    pos = torch.zeros(64, dtype=torch.int32, device=DEV)
    q = torch.zeros((64, 32, D), dtype=torch.bfloat16, device=DEV)
    k = torch.zeros((64, 8, D), dtype=torch.bfloat16, device=DEV)
    r = K.Rotary(_freq(64).to(DEV), n_q_heads=32, n_kv_heads=8, kv_dtype=torch.bfloat16, q_weight=torch.ones(D, dtype=torch.bfloat16, device=DEV))
    qo, ko, q2, k2 = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)
    r.apply(pos, q, k, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        r.apply(pos, q, k, q_out=qo, k_out=ko)
    for i in range(4):
        q.normal_()
        k.normal_()
        pos.copy_(i32(np.arange(64) * 777 + i))
        graph.replay()
        r.apply(pos, q, k, q_out=q2, k_out=k2)
        torch.cuda.synchronize()
        assert torch.equal(qo, q2) and torch.equal(ko, k2), i
