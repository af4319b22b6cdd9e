"""Refusals of plans of shared pages and of attention by them, and their oracle by hand (CPU)."""
import ctypes as C

import numpy as np
import pytest

from oracle import pages as P

tadm = pytest.importorskip("paper_2609_37924_amd")
torch = pytest.importorskip("torch")

BUF = np.zeros(4096, dtype=np.uint8)
BASE = (BUF.ctypes.data + 15) // 16 * 16  # aligned addresses that no call may follow
INV = tadm.TADM_ERR_INVALID


def rows(**kw):
    r = dict(table_dev=BASE, len_dev=None, n_dev=None, B=2, max_pages=4, len=100)
    r.update(kw)
    return tadm.tadm_page_rows(**r)


def plan(**kw):
    p = dict(data_dev=BASE, bytes=1 << 20)
    p.update(kw)
    return tadm.tadm_page_plan(**p)


@pytest.mark.parametrize("r, p, n, least, lead, says", [
    (dict(table_dev=None), {}, 3, 1, 0, "table"),
    (dict(B=0), {}, 3, 1, 0, "B=0"),
    (dict(B=1025), {}, 3, 1, 0, "B=1025"),
    (dict(len=257), {}, 3, 1, 0, "257 positions with 4 pages"),
    ({}, dict(data_dev=None), 3, 1, 0, "null plan"),
    ({}, dict(data_dev=BASE + 8), 3, 1, 0, "aligned"),
    ({}, {}, 3, 0, 0, "min_pages=0"),
    ({}, {}, 0, 1, 0, "n=0"),
    ({}, {}, 3, 1, 2, "aligned"),
    ({}, {}, 3, 1, None, "null model"),
])
def test_share_names_the_wrong_argument(r, p, n, least, lead, says):
    """lead: where the outputs begin, from an aligned address."""
    lead = None if lead is None else BASE + lead
    assert tadm.lib.tadm_pages_share(None, C.byref(rows(**r)), n, least, C.byref(plan(**p)), lead, lead) == INV
    assert says in tadm.last_error(), tadm.last_error()


@pytest.mark.parametrize("kw, says", [
    (dict(p=None), "null plan"),
    (dict(q=None), "null queries"),
    (dict(o=None), "null queries or output"),
    (dict(o=BASE + 8), "aligned"),
    (dict(lse=BASE + 2), "aligned"),
    (dict(vt=None), "null keys"),
    (dict(cap=96), "cap=96"),
    (dict(n=0), "n=0"),
    (dict(layer=2), "layer 2 of 2"),
    (dict(k=None, vt=None, cap=0), "null model"),
])
def test_attend_shared_names_the_wrong_argument(kw, says):
    a = dict(layer=1, p=C.byref(plan(B=2, max_pages=4, len=100, n=3)), q=BASE, n=3, k=BASE, vt=BASE, cap=64, o=BASE, lse=BASE)
    a.update(kw)
    pages = tadm.tadm_pages(data=BASE, scale=BASE, n_pages=8, n_layers=2, n_kv_heads=2, head_dim=16)
    assert tadm.lib.tadm_pages_attend_shared(None, C.byref(pages), a["layer"], C.byref(rows()), a["p"], a["q"], a["n"], a["k"],
                                             a["vt"], a["cap"], a["o"], a["lse"], BASE, 1 << 20) == INV
    assert says in tadm.last_error(), tadm.last_error()


def test_null_handles_and_descriptors():
    assert tadm.lib.tadm_pages_plan_bytes(None, C.byref(rows()), 1) == 0
    assert tadm.lib.tadm_pages_attend_shared_work(None, C.byref(rows()), 1) == 0
    assert tadm.lib.tadm_pages_share(None, None, 1, 1, None, None, None) == INV
    assert tadm.lib.tadm_context_share(None, 1) == INV
    with pytest.raises(ValueError):
        tadm.page_plan(torch.zeros(8, 8)[:, ::2])
    r = tadm.page_rows(torch.zeros(2, 4, dtype=torch.int32), 100)
    for bad in (torch.zeros(2), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            tadm.tadm_pages_share(None, r, 1, 1, tadm.page_plan(torch.zeros(64)), bad)


def test_groups_by_hand():
    t = [[1, 2, 3, 9], [1, 2, 3, 8], [1, 2, 7, 8], [4, 2, 7, 8], [4, 2, 7, 8], [4, 2, 7, 8]]
    full = [256] * 6
    assert P.groups(t, full) == ([0, 0, 0, 3, 3, 3], [2, 2, 2, 4, 4, 4])
    assert P.groups(t, full, 3) == ([0, 0, 2, 3, 3, 3], [3, 3, 0, 4, 4, 4])
    assert P.groups(t, [256, 256, 256, 256, 191, 256]) == ([0, 0, 0, 3, 3, 3], [2, 2, 2, 2, 2, 2])
    assert P.groups(t, [63, 256, 256, 256, 0, 256]) == ([0, 1, 1, 3, 4, 5], [0, 2, 2, 0, 0, 0])
    assert P.groups([[5]], [64]) == ([0], [0])
