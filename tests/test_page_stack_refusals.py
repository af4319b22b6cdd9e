"""Refusals of the calls on a stack of free pages, and what their oracle does by hand (CPU)."""
import ctypes as C

import numpy as np
import pytest

from oracle import pages as P

tadm = pytest.importorskip("paper_2609_37924_amd")
torch = pytest.importorskip("torch")

BUF = np.zeros(4096, dtype=np.uint8)
BASE = (BUF.ctypes.data + 15) // 16 * 16  # aligned addresses that no call may follow
INV = tadm.TADM_ERR_INVALID


def call(name, st=(), r=(), n=3, granted=BASE, slots=BASE, m=None):
    stack = dict(id_dev=BASE, state_dev=BASE, size=8)
    stack.update(st)
    rows = dict(table_dev=BASE, len_dev=None, n_dev=None, B=2, max_pages=4, len=100)
    rows.update(r)
    stack, rows = C.byref(tadm.tadm_page_stack(**stack)), C.byref(tadm.tadm_page_rows(**rows))
    if name == "assign":
        return tadm.lib.tadm_pages_assign(m, stack, rows, n, granted, slots)
    return tadm.lib.tadm_pages_release(m, stack, rows, n)


@pytest.mark.parametrize("name", ["assign", "release"])
@pytest.mark.parametrize("st, r, n, says", [
    (dict(id_dev=None), {}, 3, "null stack"),
    (dict(state_dev=None), {}, 3, "null stack"),
    (dict(size=0), {}, 3, "0 pages"),
    (dict(id_dev=BASE + 2), {}, 3, "aligned"),
    (dict(state_dev=BASE + 4), {}, 3, "state not to 8"),
    ({}, dict(table_dev=None), 3, "table"),
    ({}, dict(B=0), 3, "B=0"),
    ({}, dict(B=4097), 3, "B=4097"),
    ({}, dict(max_pages=0), 3, "max_pages"),
    ({}, dict(len=257), 3, "257 positions with 4 pages"),
    ({}, dict(len_dev=BASE + 2), 3, "aligned"),
    ({}, {}, 0, "n=0"),
    ({}, {}, (1 << 26) + 1, "n=67108865"),
    ({}, dict(B=4096), 1 << 15, "too many"),
    ({}, {}, 3, "null model"),
])
def test_calls_name_the_wrong_argument(name, st, r, n, says):
    assert call(name, st, r, n) == INV
    assert says in tadm.last_error(), tadm.last_error()


def test_outputs_of_assign():
    assert call("assign", granted=None) == INV and "granted" in tadm.last_error()
    assert call("assign", granted=BASE + 2) == INV and "aligned" in tadm.last_error()
    assert call("assign", slots=BASE + 4) == INV and "aligned" in tadm.last_error()
    assert call("assign", slots=None) == INV and "null model" in tadm.last_error()
    assert tadm.lib.tadm_pages_assign(None, None, None, 1, BASE, None) == INV
    assert tadm.lib.tadm_pages_release(None, None, None, 1) == INV


@pytest.mark.parametrize("name", ["n_dev", "len_dev"])
@pytest.mark.parametrize("by", [-4, 0, 4])
def test_assign_refuses_to_write_over_its_lengths(name, by):
    """Blocks read the lengths of the rows before theirs while others write what was granted (B=2: 8 bytes each)."""
    at = BASE + 64
    assert call("assign", r={name: at}, granted=at + by) == INV
    assert "granted_dev" in tadm.last_error() and name in tadm.last_error(), tadm.last_error()
    for clear in (-8, 8):
        assert call("assign", r={name: at}, granted=at + clear) == INV and "null model" in tadm.last_error()


def test_descriptors_refuse_other_tensors():
    ids, state = torch.zeros(8, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    assert tadm.page_stack(ids, state).size == 8
    for bad in ((ids.long(), state), (ids, state.float()), (ids, state[:3]), (ids[::2], state), (ids.view(2, 4), state)):
        with pytest.raises(ValueError):
            tadm.page_stack(*bad)
    st = tadm.page_stack(ids, state)
    rows = tadm.page_rows(torch.zeros(2, 4, dtype=torch.int32), 100)
    for granted, slots in ((state[:3], None), (state[:2].long(), None), (state[:2], torch.zeros(2, 3, dtype=torch.int32)),
                           (state[:2], torch.zeros(2, 4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            tadm.tadm_pages_assign(None, st, rows, 3, granted, slots)


def test_oracle_by_hand():
    table = [[5, -1, -1], [-1, -1, -1], [6, -1, -1], [-1, -1, -1]]
    ids = [0, 1, 2, 3, -1, -1, -1, -1]
    granted, slots, free = P.assign(table, [60, 0, 10, 64], [5, 129, 3, 1], ids, 4, 8)
    # row 0 takes page 3; row 1 the other three; row 2 needs none; row 3 has to wait
    assert granted == [5, 129, 3, 0] and free == 0
    assert table == [[5, 3, -1], [2, 1, 0], [6, -1, -1], [-1, -1, -1]]
    assert slots[0] == [5 * 64 + 60, 5 * 64 + 61, 5 * 64 + 62, 5 * 64 + 63, 3 * 64] and slots[1][128] == 0
    assert slots[2] == [6 * 64 + 10, 6 * 64 + 11, 6 * 64 + 12] and slots[3] == []
    free = P.release(table, [60, 0, 10, 64], granted, ids, free, 8)
    assert free == 4 and ids[:4] == [3, 2, 1, 0]
    assert table == [[5, -1, -1], [-1, -1, -1], [6, -1, -1], [-1, -1, -1]]
