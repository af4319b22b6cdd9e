"""Refusals of the page operators, the pool and pooled contexts (CPU).

The operators check their arguments before the model, so each wrong argument of a call
without a model is named in the error; nothing reaches a device."""
import ctypes as C

import numpy as np
import pytest

tadm = pytest.importorskip("paper_2609_37924_amd")

BUF = np.zeros(4096, dtype=np.uint8)
BASE = (BUF.ctypes.data + 15) // 16 * 16  # aligned addresses that no call may follow
INV = tadm.TADM_ERR_INVALID


def pages(**kw):
    p = dict(data=BASE, scale=BASE, n_pages=8, n_layers=2, n_kv_heads=2, head_dim=16)
    p.update(kw)
    return tadm.tadm_pages(**p)


def rows(**kw):
    r = dict(table_dev=BASE, len_dev=None, n_dev=None, B=2, max_pages=4, len=100)
    r.update(kw)
    return tadm.tadm_page_rows(**r)


def call(name, p=None, r=None, m=None, **kw):
    p, r = C.byref(p if p is not None else pages()), C.byref(r if r is not None else rows())
    a = dict(layer=1, k=BASE, vt=BASE, n=3, cap=64, q=BASE, o=BASE, lse=BASE, work=BASE, bytes=1 << 20)
    a.update(kw)
    if name == "append":
        return tadm.lib.tadm_pages_append(m, p, a["layer"], r, a["k"], a["vt"], a["n"], a["cap"])
    if name == "read":
        return tadm.lib.tadm_pages_read(m, p, a["layer"], r, a["k"], a["vt"], a["cap"])
    return tadm.lib.tadm_pages_attend(m, p, a["layer"], r, a["q"], a["n"], a["k"], a["vt"], a["cap"], a["o"], a["lse"],
                                      a["work"], a["bytes"])


@pytest.mark.parametrize("name", ["append", "attend", "read"])
@pytest.mark.parametrize("p, r, kw, says", [
    (dict(data=None), {}, {}, "null pages"),
    (dict(scale=None), {}, {}, "null pages"),
    (dict(n_pages=0), {}, {}, "0 pages"),
    (dict(n_layers=0), {}, {}, "0 layers"),
    (dict(head_dim=0), {}, {}, "heads x 0"),
    (dict(data=BASE + 4), {}, {}, "aligned"),
    ({}, {}, dict(layer=2), "layer 2 of 2"),
    ({}, {}, dict(layer=-1), "layer -1"),
    ({}, dict(table_dev=None), {}, "table"),
    ({}, dict(B=0), {}, "B=0"),
    ({}, dict(B=65536), {}, "B=65536"),
    ({}, dict(max_pages=0), {}, "max_pages"),
    ({}, dict(len=-1), {}, "-1 positions"),
    ({}, dict(len=257), {}, "257 positions with 4 pages"),
    ({}, dict(len_dev=BASE + 2), {}, "aligned"),
    ({}, dict(n_dev=BASE + 1), {}, "aligned"),
    ({}, {}, dict(vt=None), "null keys"),
    ({}, {}, dict(cap=96), "cap=96"),
    ({}, dict(len=65), dict(n=65, cap=64), "cap=64"),
    ({}, {}, dict(k=BASE + 8, cap=128), "aligned"),
    ({}, {}, dict(cap=128), "null model"),
])
def test_operators_name_the_wrong_argument(name, p, r, kw, says):
    assert call(name, pages(**p), rows(**r), **kw) == INV
    assert says in tadm.last_error(), tadm.last_error()


@pytest.mark.parametrize("name, r, kw, says", [
    ("append", {}, dict(n=0), "n=0"),
    ("append", dict(len=250), dict(n=7), "[250, 257) with 4 pages"),
    ("append", {}, dict(k=None, vt=None), "null keys"),
    ("attend", {}, dict(n=0), "n=0"),
    ("attend", {}, dict(n=-5), "n=-5"),
    ("attend", {}, dict(q=None), "null queries"),
    ("attend", {}, dict(o=None), "null queries or output"),
    ("attend", {}, dict(o=BASE + 8), "aligned"),
    ("attend", {}, dict(k=None, vt=None, cap=0), "null model"),  # no window keys: cap is not looked at
    ("append", dict(len=250, len_dev=BASE), dict(n=7), "null model"),  # lengths on the device: cut there
])
def test_operators_of_one_kind(name, r, kw, says):
    assert call(name, None, rows(**r), **kw) == INV
    assert says in tadm.last_error(), tadm.last_error()


@pytest.mark.parametrize("src, dst, says", [
    ([0], [8], "destination outside"),
    ([0], [-1], "destination outside"),
    ([8], [0], "source page 8"),
    ([-1], [0], "source page -1"),
    ([0, 1], [2, 2], "twice"),
    ([0, 1], [2, 0], "source and a destination"),
    ([3], [3], "source and a destination"),
    ([0] * 9, list(range(9)), "9 copies"),
    ([0, 0], [1, 2], "null model"),
    ([], [], "null model"),
])
def test_copy_lists(src, dst, says):
    a, b = (np.array(x, dtype=np.int32) for x in (src, dst))
    assert tadm.lib.tadm_pages_copy(None, C.byref(pages()), a.ctypes.data, b.ctypes.data, len(src)) == INV
    assert says in tadm.last_error(), tadm.last_error()


def test_copy_counts():
    assert tadm.lib.tadm_pages_copy(None, C.byref(pages()), None, None, 1) == INV and "null page list" in tadm.last_error()
    assert tadm.lib.tadm_pages_copy(None, C.byref(pages()), BASE, BASE, -1) == INV and "-1 copies" in tadm.last_error()
    assert tadm.lib.tadm_pages_copy(None, None, BASE, BASE, 1) == INV


def test_null_handles():
    out = C.c_void_p()
    lib = tadm.lib
    assert lib.tadm_pages_attend_work(None, C.byref(rows()), 1) == 0
    assert lib.tadm_pages_attend_work(None, None, 1) == 0
    assert lib.tadm_pool_create(None, 4, C.byref(out)) == INV
    assert lib.tadm_pool_destroy(None) == INV
    assert lib.tadm_pool_size(None) == 0 and lib.tadm_pool_free_pages(None) == 0
    assert lib.tadm_pool_pages(None, C.byref(pages())) == INV
    assert lib.tadm_pool_compact(None) == INV
    assert lib.tadm_pool_resize(None, 4) == INV
    assert lib.tadm_context_create_pooled(None, None, 1, 64, C.byref(out)) == INV
    assert lib.tadm_context_fork(None, BASE, 1, C.byref(out)) == INV
    assert lib.tadm_context_truncate(None, 0) == INV
    assert lib.tadm_context_rows(None, C.byref(rows())) == INV


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    data, scale = torch.zeros(4, 2, 3, 2, 64 * 16, dtype=torch.uint8), torch.zeros(4, 2, 3, 2)
    p = tadm.page_set(data, scale)
    assert (p.n_pages, p.n_layers, p.n_kv_heads, p.head_dim) == (4, 2, 3, 16)
    for d, s in ((data[..., :100], scale), (data, scale[:2]), (data.float(), scale), (data, scale.half()),
                 (data.transpose(0, 1), scale.transpose(0, 1))):
        with pytest.raises(ValueError):
            tadm.page_set(d, s)
    with pytest.raises(ValueError):
        tadm.tadm_pages_copy(None, p, [1, 2], [3])


@pytest.mark.parametrize("name", ["append", "attend"])
@pytest.mark.parametrize("B, n", [(1, (1 << 26) + 1), (1, 2**31 - 64), (65535, 1025)])
def test_windows_beyond_a_launch(name, B, n):
    r = rows(B=B, max_pages=1 << 24, len=0)
    assert call(name, r=r, n=n, cap=2**31 - 64) == INV
    assert "2^26" in tadm.last_error()


def test_binding_refuses_wrong_tables():
    torch = pytest.importorskip("torch")
    table, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    r = tadm.page_rows(table, 100, lens, lens)
    assert (r.B, r.max_pages, r.len) == (3, 4, 100)
    for bad in (table.long(), table[:, ::2], table.T, table[0], table.float()):
        with pytest.raises(ValueError):
            tadm.page_rows(bad, 100)
    for bad in (lens.long(), lens[:2], torch.zeros(6, dtype=torch.int32)[::2], lens[:, None]):
        with pytest.raises(ValueError):
            tadm.page_rows(table, 100, bad)
        with pytest.raises(ValueError):
            tadm.page_rows(table, 100, None, bad)
