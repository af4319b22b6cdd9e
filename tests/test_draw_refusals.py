"""Refusals of draws from given numbers (CPU)."""
import ctypes as C

import numpy as np
import pytest

tadm = pytest.importorskip("paper_2609_37924_amd")
torch = pytest.importorskip("torch")

BUF = np.zeros(4096, dtype=np.uint8)
BASE = (BUF.ctypes.data + 15) // 16 * 16  # aligned addresses that no call may follow


def call(set_=None, **kw):
    a = dict(m=None, logits=BASE, ld=64, R=2, u=BASE, token=BASE, logp=BASE, work=BASE, bytes=1 << 20)
    a.update(kw)
    s = None if set_ is None else C.byref(tadm.tadm_row_settings(**set_))
    return tadm.lib.tadm_sample_rows(a["m"], a["logits"], a["ld"], a["R"], s, a["u"], a["token"], a["logp"], a["work"], a["bytes"])


@pytest.mark.parametrize("kw, set_, says", [
    (dict(logits=None), None, "null logits"),
    (dict(u=None), None, "null logits, u_dev"),
    (dict(token=None), None, "token_dev"),
    (dict(R=0), None, "R=0"),
    (dict(R=(1 << 21) + 1), None, "R=2097153"),
    (dict(logits=BASE + 2), None, "aligned"),
    (dict(logp=BASE + 1), None, "aligned"),
    ({}, dict(temperature_dev=BASE + 2), "aligned"),
    ({}, dict(top_k_dev=BASE + 2), "aligned"),
    ({}, dict(top_p_dev=BASE + 2), "aligned"),
    ({}, dict(min_p_dev=BASE + 2), "aligned"),
    (dict(logp=None, work=None), None, "null model"),
])
def test_calls_name_the_wrong_argument(kw, set_, says):
    assert call(set_, **kw) == tadm.TADM_ERR_INVALID
    assert says in tadm.last_error(), tadm.last_error()


def test_null_model_needs_no_scratch():
    assert tadm.tadm_sample_rows_work(None, 4) == 0


def test_binding_refuses_other_tensors():
    f, i = torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        tadm.row_settings(temperature=f.double())
    with pytest.raises(ValueError):
        tadm.row_settings(top_k=f)
    with pytest.raises(ValueError):
        tadm.row_settings(top_p=torch.zeros(6)[::2])
    logits = torch.zeros(3, 8)
    ok = tadm.row_settings(top_p=f)
    for args in ((logits.double(), ok, f, i), (logits.t(), ok, f, i), (logits, ok, f[:2], i), (logits, ok, f, f),
                 (logits, ok, f, i, i), (logits, tadm.row_settings(top_p=torch.zeros(4)), f, i)):
        with pytest.raises(ValueError):
            tadm.tadm_sample_rows(None, *args)
    with pytest.raises(tadm.TadmError):
        tadm.tadm_sample_rows(None, logits, ok, f, i)
