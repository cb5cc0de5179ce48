"""Refusals of the 8-bit paged cache's calls, which come before any device is touched.  No GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2605_18071_amd import kvd

P = 4096                                                  # a non-null, aligned address: never dereferenced here


def _rows(**kw):
    a = dict(n_seqs=2, max_pages=8, n_rows=4, max_runs=4, page_size=16, n_blocks=10, page_table=P, kv_len=2 * P, row_start=3 * P,
             row_seq=4 * P, row_pos=5 * P, runs=6 * P, counts=7 * P)
    a.update(kw)
    return kvd.KvdQ8Rows(**a)


def _cache(**kw):
    a = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_blocks=10, sink_pages=0, recent_pages=0, kv_dtype=kvd.KVD_BF16,
             softmax_scale=0.0, pages=P, exps=P, means=P, mean_scales=P)
    a.update(kw)
    return kvd.KvdQ8Cache(**a)


BAD_ROWS = [dict(n_seqs=0), dict(n_seqs=4097), dict(max_pages=0), dict(max_pages=65537), dict(n_rows=0), dict(n_rows=131073),
            dict(max_runs=0), dict(max_runs=131073), dict(page_size=0), dict(page_size=8), dict(page_size=24), dict(page_size=272),
            dict(n_blocks=0)]


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_sizes_of_the_rows(kw):
    lib = kvd.load()
    r, c = _rows(**kw), _cache()
    assert lib.kvd_q8_map(C.byref(r), P, 8 * P, P, 4, P, None) == kvd.ERR_SHAPE
    assert lib.kvd_q8_append(C.byref(c), C.byref(r), P, 256, P, 256, None) == kvd.ERR_SHAPE
    assert lib.kvd_q8_workspace_bytes(C.byref(c), C.byref(r), 0) == kvd.ERR_SHAPE
    assert lib.kvd_q8_select(C.byref(c), C.byref(r), P, 1024, P, 4, P, 1 << 40, None) == kvd.ERR_SHAPE
    assert lib.kvd_q8_attn(C.byref(c), C.byref(r), P, 1024, None, 0, P, None, P, 1 << 40, None) == kvd.ERR_SHAPE


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=64), kvd.ERR_SHAPE), (dict(n_q_heads=7), kvd.ERR_SHAPE), (dict(n_q_heads=18), kvd.ERR_SHAPE),
    (dict(n_q_heads=0), kvd.ERR_SHAPE), (dict(n_kv_heads=0), kvd.ERR_SHAPE), (dict(n_q_heads=514, n_kv_heads=257), kvd.ERR_SHAPE),
    (dict(page_size=32), kvd.ERR_SHAPE), (dict(n_blocks=11), kvd.ERR_SHAPE), (dict(sink_pages=-1), kvd.ERR_SHAPE),
    (dict(recent_pages=-1), kvd.ERR_SHAPE), (dict(kv_dtype=2), kvd.ERR_DTYPE), (dict(softmax_scale=float("nan")), kvd.ERR_ARG),
    (dict(softmax_scale=-1.0), kvd.ERR_ARG), (dict(softmax_scale=float("inf")), kvd.ERR_ARG),
])
def test_settings_of_the_cache(kw, want):
    lib = kvd.load()
    r, c = _rows(), _cache(**kw)
    assert lib.kvd_q8_append(C.byref(c), C.byref(r), P, 1 << 20, P, 1 << 20, None) == want
    assert lib.kvd_q8_workspace_bytes(C.byref(c), C.byref(r), 1) == want
    assert lib.kvd_q8_select(C.byref(c), C.byref(r), P, 1 << 20, P, 4, P, 1 << 40, None) == want
    assert lib.kvd_q8_attn(C.byref(c), C.byref(r), P, 1 << 20, None, 0, P, None, P, 1 << 40, None) == want


def test_pointers_strides_and_workspaces():
    lib = kvd.load()
    r, c = _rows(), _cache()
    br, bc = C.byref(r), C.byref(c)

    def map_(rows=br, lens=P, new=8 * P, free=P, n=4, count=P):
        return lib.kvd_q8_map(rows, lens, new, free, n, count, None)

    assert map_(rows=None) == map_(lens=None) == map_(new=None) == map_(free=None) == map_(count=None) == kvd.ERR_ARG
    assert map_(lens=2 * P) == map_(new=2 * P) == map_(count=7 * P + 12) == kvd.ERR_ARG      # read by some while others write it
    assert map_(n=-1) == kvd.ERR_SHAPE and map_(lens=P + 2) == kvd.ERR_ARG
    for name in ("page_table", "kv_len", "row_start", "row_seq", "row_pos", "runs", "counts"):
        assert map_(rows=C.byref(_rows(**{name: None}))) == kvd.ERR_ARG
    assert map_(rows=C.byref(_rows(runs=P + 4))) == kvd.ERR_ARG

    def append(cache=bc, rows=br, k=P, ks=256, v=P, vs=256):
        return lib.kvd_q8_append(cache, rows, k, ks, v, vs, None)

    assert append(cache=None) == append(rows=None) == append(k=None) == append(v=None) == append(k=P + 8) == kvd.ERR_ARG
    assert append(ks=255) == append(vs=252) == append(ks=260) == append(vs=-256) == kvd.ERR_SHAPE
    for name in ("pages", "exps", "means", "mean_scales"):
        assert append(cache=C.byref(_cache(**{name: None}))) == kvd.ERR_ARG
    assert append(rows=C.byref(_rows(runs=None))) == kvd.ERR_ARG and append(cache=C.byref(_cache(exps=P + 1))) == kvd.ERR_ARG

    need = lib.kvd_q8_workspace_bytes(bc, br, 1)
    assert need >= 4 * 2 * 8 * 4

    def select(cache=bc, rows=br, q=P, qs=1024, sel=P, k=4, ws=P, n=need):
        return lib.kvd_q8_select(cache, rows, q, qs, sel, k, ws, n, None)

    assert select(cache=None) == select(rows=None) == select(q=None) == select(sel=None) == select(ws=None) == kvd.ERR_ARG
    assert select(q=P + 2) == select(ws=P + 4) == select(rows=C.byref(_rows(row_pos=None))) == kvd.ERR_ARG
    assert select(k=0) == select(k=2049) == select(qs=1016) == select(qs=1028) == kvd.ERR_SHAPE
    assert select(n=need - 1) == select(cache=C.byref(_cache(sink_pages=3, recent_pages=2))) == kvd.ERR_CAPACITY
    assert select(cache=C.byref(_cache(sink_pages=2 ** 31 - 1, recent_pages=2 ** 31 - 1))) == kvd.ERR_CAPACITY

    need = lib.kvd_q8_workspace_bytes(bc, br, 0)

    def attn(cache=bc, rows=br, q=P, qs=1024, sel=None, k=0, out=8 * P, lse=None, ws=P, n=need):
        return lib.kvd_q8_attn(cache, rows, q, qs, sel, k, out, lse, ws, n, None)

    assert attn(cache=None) == attn(rows=None) == attn(q=None) == attn(out=None) == attn(ws=None) == kvd.ERR_ARG
    assert attn(out=P) == kvd.ERR_ARG                     # in place: pieces of a row still read what others write
    assert attn(out=P + 8) == attn(lse=P + 1) == attn(sel=P + 2, k=4) == attn(rows=C.byref(_rows(kv_len=None))) == kvd.ERR_ARG
    assert attn(qs=0) == attn(sel=P, k=0) == attn(sel=P, k=2049) == kvd.ERR_SHAPE
    assert attn(n=need - 1) == kvd.ERR_CAPACITY


def test_the_binding_refuses_before_the_library():
    table = torch.zeros((2, 8), dtype=torch.int32)
    rows = kvd.Q8Rows(table, page_size=16, n_blocks=10, n_rows=4)
    cache = kvd.Q8Cache(n_blocks=10, n_q_heads=8, n_kv_heads=2, page_size=16, kv_dtype=torch.bfloat16, device="cpu")
    i2, one = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    q = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    ws = cache.workspace(rows)
    for call in (lambda: rows.map(i2, i2, i2, one), lambda: cache.append(rows, k, k), lambda: cache.attend(rows, q, q.clone(), ws)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="seq_len"):
        rows.map(i2.long(), i2, i2, one)
    with pytest.raises(ValueError, match="n_new"):
        rows.map(i2, one, i2, one)
    with pytest.raises(ValueError, match="k_new"):
        cache.append(rows, k[:3], k)
    with pytest.raises(ValueError, match="v_new"):
        cache.append(rows, k, k.half())
    with pytest.raises(ValueError, match="k_new"):
        cache.append(rows, k.transpose(1, 2).contiguous().transpose(1, 2), k)
    with pytest.raises(ValueError, match="out"):
        cache.attend(rows, q, q[:, ::2], ws)
    with pytest.raises(ValueError, match="sel_pages"):
        cache.attend(rows, q, q.clone(), ws, sel_pages=torch.zeros((4, 8, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="lse"):
        cache.attend(rows, q, q.clone(), ws, lse=torch.zeros((4, 8), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="page_table"):
        kvd.Q8Rows(table[0], page_size=16, n_blocks=10, n_rows=4)
    with pytest.raises(ValueError, match="runs"):
        kvd.Q8Rows(table, page_size=16, n_blocks=10, n_rows=4, runs=torch.zeros((4, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="pages"):
        kvd.Q8Cache(n_blocks=9, n_q_heads=8, n_kv_heads=2, page_size=16, kv_dtype=torch.bfloat16, buffers=dict(pages=cache.pages))
    with pytest.raises(ValueError, match="buffers"):
        kvd.Q8Cache(n_blocks=9, n_q_heads=8, n_kv_heads=2, page_size=16, kv_dtype=torch.bfloat16, buffers=dict(keys=cache.pages))
    with pytest.raises(kvd.KvdError):
        kvd.Q8Cache(n_blocks=10, n_q_heads=18, n_kv_heads=2, page_size=16, kv_dtype=torch.float16, device="cpu").workspace(rows)
