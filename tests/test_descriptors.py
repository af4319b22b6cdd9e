"""Descriptors hold the tensors whose addresses they have (CPU): one made of temporaries is no use of freed memory."""
import ctypes as C
import gc
import weakref

import pytest

torch = pytest.importorskip("torch")
tadm = pytest.importorskip("paper_2609_37924_amd")


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


MAKE = {
    "pages": lambda keep: tadm.page_set(keep(torch.zeros(4, 2, 3, 2, 64 * 16, dtype=torch.uint8)), keep(torch.zeros(4, 2, 3, 2))),
    "rows": lambda keep: tadm.page_rows(keep(i32(2, 4)), 100, keep(i32(2)), keep(i32(2))),
    "rows without lengths": lambda keep: tadm.page_rows(keep(i32(2, 4)), 100),
    "plan": lambda keep: tadm.page_plan(keep(torch.zeros(512, dtype=torch.uint8))),
    "stack": lambda keep: tadm.page_stack(keep(i32(8)), keep(i32(4))),
    "settings": lambda keep: tadm.row_settings(keep(torch.zeros(3)), keep(i32(3)), keep(torch.zeros(3)), keep(torch.zeros(3))),
    "one setting": lambda keep: tadm.row_settings(top_p=keep(torch.zeros(3))),
}


@pytest.mark.parametrize("name", list(MAKE))
def test_a_descriptor_of_temporaries(name):
    at, alive = [], []

    def keep(t):
        at.append(t.data_ptr())
        alive.append(weakref.ref(t))
        return t

    d = MAKE[name](keep)
    gc.collect()
    assert all(r() is not None for r in alive)
    held = [getattr(d, f) for f, kind in d._fields_ if kind is C.c_void_p]
    assert [a for a in held if a] == at
    del d
    gc.collect()
    assert all(r() is None for r in alive)  # and no longer than they are needed
