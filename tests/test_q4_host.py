"""Refusals of the 4-bit paged cache's calls and of the rotation, which come before any device is touched.  No GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2605_18071_amd import kvd
from tests.test_q8_host import BAD_ROWS, P, _rows


def _cache(**kw):
    a = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_blocks=10, kv_dtype=kvd.KVD_BF16, softmax_scale=0.0, pages=P)
    a.update(kw)
    return kvd.KvdQ4Cache(**a)


def _calls(lib, c, r):
    c, r = C.byref(c), C.byref(r)
    return [lib.kvd_q4_append(c, r, P, 1 << 20, P, 1 << 20, None), lib.kvd_q4_read(c, r, P, 1 << 20, P, 1 << 20, None),
            lib.kvd_q4_workspace_bytes(c, r), lib.kvd_q4_attn(c, r, P, 1 << 20, None, 8 * P, None, P, 1 << 40, None)]


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_sizes_of_the_rows(kw):
    assert _calls(kvd.load(), _cache(), _rows(**kw)) == [kvd.ERR_SHAPE] * 4


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=64), kvd.ERR_SHAPE), (dict(n_q_heads=7), kvd.ERR_SHAPE), (dict(n_q_heads=18), kvd.ERR_SHAPE),
    (dict(n_q_heads=0), kvd.ERR_SHAPE), (dict(n_kv_heads=0), kvd.ERR_SHAPE), (dict(n_q_heads=514, n_kv_heads=257), kvd.ERR_SHAPE),
    (dict(page_size=32), kvd.ERR_SHAPE), (dict(n_blocks=11), kvd.ERR_SHAPE), (dict(kv_dtype=2), kvd.ERR_DTYPE),
    (dict(softmax_scale=float("nan")), kvd.ERR_ARG), (dict(softmax_scale=-1.0), kvd.ERR_ARG), (dict(softmax_scale=float("inf")), kvd.ERR_ARG),
])
def test_settings_of_the_cache(kw, want):
    assert _calls(kvd.load(), _cache(**kw), _rows()) == [want] * 4


def test_a_pool_whose_lines_need_more_than_32_bits():
    # 17 lines a tile, 256 heads: 986895 tiles of a head are the most
    lib = kvd.load()
    for n, want in ((986895, True), (986896, False)):
        c, r = _cache(n_blocks=n, n_kv_heads=256, n_q_heads=256), _rows(n_blocks=n)
        assert (lib.kvd_q4_workspace_bytes(C.byref(c), C.byref(r)) > 0) == want


def test_pointers_strides_and_workspaces():
    lib = kvd.load()
    br, bc = C.byref(_rows()), C.byref(_cache())
    for fn in (lib.kvd_q4_append, lib.kvd_q4_read):
        def call(cache=bc, rows=br, k=P, ks=256, v=P, vs=256):
            return fn(cache, rows, k, ks, v, vs, None)

        assert call(cache=None) == call(rows=None) == call(k=None) == call(v=None) == call(k=P + 8) == kvd.ERR_ARG
        assert call(ks=255) == call(vs=252) == call(ks=260) == call(vs=-256) == kvd.ERR_SHAPE
        assert call(cache=C.byref(_cache(pages=None))) == call(cache=C.byref(_cache(pages=P + 64))) == kvd.ERR_ARG
    assert lib.kvd_q4_append(bc, C.byref(_rows(runs=P + 4)), P, 256, P, 256, None) == kvd.ERR_ARG
    for name in ("page_table", "row_seq", "row_pos"):
        assert lib.kvd_q4_read(bc, C.byref(_rows(**{name: None})), P, 256, P, 256, None) == kvd.ERR_ARG

    need = lib.kvd_q4_workspace_bytes(bc, br)
    assert need > 8192

    def attn(cache=bc, rows=br, q=P, qs=1024, scores=None, out=8 * P, lse=None, ws=P, n=need):
        return lib.kvd_q4_attn(cache, rows, q, qs, scores, out, lse, ws, n, None)

    assert attn(cache=None) == attn(rows=None) == attn(q=None) == attn(out=None) == attn(ws=None) == kvd.ERR_ARG
    assert attn(out=P) == attn(out=P + 8) == attn(lse=P + 1) == attn(ws=P + 8) == kvd.ERR_ARG
    for name in ("page_table", "kv_len", "row_start"):
        assert attn(rows=C.byref(_rows(**{name: None}))) == kvd.ERR_ARG
    assert attn(qs=0) == attn(qs=1028) == kvd.ERR_SHAPE and attn(n=need - 1) == kvd.ERR_CAPACITY

    def scores(cap=0.0, window=0, slopes=None, row_from=None, prefix_len=None):
        return attn(scores=C.byref(kvd.KvdQ4Scores(cap, window, slopes, row_from, prefix_len)), n=0)

    assert scores() == scores(cap=30.0, window=9, slopes=P, row_from=P, prefix_len=P) == kvd.ERR_CAPACITY    # nothing but the workspace is wrong
    assert scores(cap=-1.0) == scores(cap=float("nan")) == scores(cap=float("inf")) == scores(cap=1e-45) == scores(cap=1e29) == kvd.ERR_ARG
    assert scores(window=-1) == kvd.ERR_SHAPE
    assert scores(slopes=P + 1) == scores(row_from=P + 2) == scores(prefix_len=P + 3) == kvd.ERR_ARG


def _rotary(pairs=(64, 0, 0, 0), **kw):
    a = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, kv_dtype=kvd.KVD_F16, rot_dim=128, interleaved=0, n_axes=1, axis_pairs=(C.c_int32 * 4)(*pairs),
             eps=1e-6, q_weight=None, k_weight=None, inv_freq=P)
    a.update(kw)
    return kvd.KvdRotary(**a)


def test_refusals_of_the_rotation():
    lib = kvd.load()

    def call(c=None, pos=P, ps=4, n=4, q=P, qs=1024, qo=2 * P, qos=1024, k=3 * P, ks=256, ko=4 * P, kos=256):
        return lib.kvd_norm_rotate(C.byref(c or _rotary()), pos, ps, n, q, qs, qo, qos, k, ks, ko, kos, None)

    assert lib.kvd_norm_rotate(None, P, 4, 4, P, 1024, P, 1024, P, 256, P, 256, None) == kvd.ERR_ARG
    assert call(_rotary(kv_dtype=2)) == kvd.ERR_DTYPE
    for bad in (dict(head_dim=64), dict(rot_dim=-16), dict(rot_dim=144), dict(rot_dim=8), dict(n_axes=0), dict(n_axes=5), dict(pairs=(63, 0, 0, 0)),
                dict(pairs=(65, 0, 0, 0)), dict(pairs=(32, 31, 0, 0), n_axes=2), dict(pairs=(-1, 65, 0, 0), n_axes=2), dict(n_q_heads=0),
                dict(n_kv_heads=-1), dict(n_q_heads=65537), dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 66, 0), n_axes=3)):
        assert call(_rotary(**bad)) == kvd.ERR_SHAPE, bad
    assert call(_rotary(pairs=(60, 4, 0, 0), n_axes=2), ps=3) == kvd.ERR_SHAPE
    assert call(n=0) == call(n=(1 << 24) + 1) == kvd.ERR_SHAPE
    assert call(qs=1016) == call(qos=1028) == call(ks=0) == call(kos=-256) == kvd.ERR_SHAPE
    assert call(_rotary(eps=-1.0)) == call(_rotary(eps=float("nan"))) == call(_rotary(eps=float("inf"))) == kvd.ERR_ARG
    assert call(pos=None) == call(pos=P + 2) == call(_rotary(inv_freq=None)) == call(q=None, k=None) == kvd.ERR_ARG
    assert call(q=P + 8) == call(qo=None) == call(k=3 * P + 2) == call(ko=4 * P + 4) == kvd.ERR_ARG
    assert call(_rotary(q_weight=P + 2)) == call(_rotary(k_weight=P + 8)) == kvd.ERR_ARG
    assert call(qo=P, qos=2048) == call(ko=3 * P, kos=512) == kvd.ERR_ARG             # in place, but rows elsewhere


def test_the_binding_refuses_before_the_library():
    table = torch.zeros((2, 8), dtype=torch.int32)
    rows = kvd.Q8Rows(table, page_size=16, n_blocks=10, n_rows=4)
    cache = kvd.Q4Cache(n_blocks=10, n_q_heads=8, n_kv_heads=2, page_size=16, kv_dtype=torch.bfloat16, device="cpu")
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    q = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    ws = cache.workspace(rows)
    rot = kvd.Rotary(torch.zeros(64), n_q_heads=8, n_kv_heads=2, kv_dtype=torch.bfloat16)
    pos = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: cache.append(rows, k, k), lambda: cache.read(rows, k, k.clone()), lambda: cache.attend(rows, q, q.clone(), ws),
                 lambda: rot.apply(pos, q, k)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for what, call in [
        ("k_new", lambda: cache.append(rows, k[:3], k)), ("v_new", lambda: cache.append(rows, k, k.half())), ("v:", lambda: cache.read(rows, k, q)),
        ("out", lambda: cache.attend(rows, q, q[:, ::2], ws)), ("lse", lambda: cache.attend(rows, q, q.clone(), ws, lse=torch.zeros(4, 2))),
        ("slopes", lambda: cache.attend(rows, q, q.clone(), ws, slopes=torch.zeros(2))),
        ("row_from", lambda: cache.attend(rows, q, q.clone(), ws, row_from=torch.zeros(4))),
        ("prefix_len", lambda: cache.attend(rows, q, q.clone(), ws, prefix_len=torch.zeros(4, dtype=torch.int32))),
        ("window", lambda: cache.attend(rows, q, q.clone(), ws, window=1 << 31)),
        ("window", lambda: cache.attend(rows, q, q.clone(), ws, window=-1)),
        ("pages", lambda: kvd.Q4Cache(n_blocks=9, n_q_heads=8, n_kv_heads=2, page_size=16, kv_dtype=torch.bfloat16, pages=cache.pages)),
        ("page_size", lambda: kvd.Q4Cache(n_blocks=9, n_q_heads=8, n_kv_heads=2, page_size=24, kv_dtype=torch.bfloat16, device="cpu")),
        ("kv_dtype", lambda: kvd.Q4Cache(n_blocks=9, n_q_heads=8, n_kv_heads=2, page_size=16, kv_dtype=torch.float32, device="cpu")),
        ("positions", lambda: rot.apply(pos.long(), q, k)), ("positions", lambda: rot.apply(pos.view(2, 2), q, k)), ("q:", lambda: rot.apply(pos, k)),
        ("wanted", lambda: rot.apply(pos, None)), ("k_out", lambda: rot.apply(pos, q, k_out=k)), ("q_out", lambda: rot.apply(pos, q, q_out=k)),
        ("axis_pairs", lambda: kvd.Rotary(torch.zeros(64), n_q_heads=8, n_kv_heads=2, kv_dtype=torch.bfloat16, axis_pairs=[32, 16])),
        ("q_weight", lambda: kvd.Rotary(torch.zeros(64), n_q_heads=8, n_kv_heads=2, kv_dtype=torch.bfloat16, q_weight=torch.zeros(128))),
        ("inv_freq", lambda: kvd.Rotary(torch.zeros(64).double(), n_q_heads=8, n_kv_heads=2, kv_dtype=torch.bfloat16)),
    ]:
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(kvd.KvdError):
        kvd.Q4Cache(n_blocks=10, n_q_heads=18, n_kv_heads=2, page_size=16, kv_dtype=torch.float16, device="cpu").workspace(rows)
