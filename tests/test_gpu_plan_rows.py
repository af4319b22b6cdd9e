"""A plan serves the rows that it was made of: calls with another table or other arrays of lengths, of the same sizes,
are refused, and descriptors made anew of the same tensors are not."""
import numpy as np
import pytest
import torch

from test_gpu_pages import model
from test_gpu_pages_shared import attend, spread, state_of

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def test_a_plan_of_other_rows_is_refused():
    m = model("bf16", 4, 4, 64)
    try:
        s = state_of(m, np.random.default_rng(1), "bf16", 4, 4, 64, [(3, spread(192, 5))], 2)
        data = torch.full((tadm.tadm_pages_plan_bytes(m, s["r"], 2),), 0xff, dtype=torch.uint8, device="cuda")
        plan, most = tadm.page_plan(data), s["mp"] * 64
        tadm.tadm_pages_share(m, s["r"], 2, 1, plan)
        attend(m, s, plan)
        want = s["o"].clone()
        others = dict(table=tadm.page_rows(s["t"].clone(), most, s["ln"], s["nn"]), lengths=tadm.page_rows(s["t"], most, s["ln"].clone(), s["nn"]),
                      tokens=tadm.page_rows(s["t"], most, s["ln"], s["nn"].clone()), no_lengths=tadm.page_rows(s["t"], most, None, s["nn"]),
                      no_tokens=tadm.page_rows(s["t"], most, s["ln"]))
        for name, r in others.items():
            with pytest.raises(tadm.TadmError, match="another table") as e:
                attend(m, dict(s, r=r), plan)
            assert e.value.status == tadm.TADM_ERR_STATE, name
        s["o"].zero_()
        attend(m, dict(s, r=tadm.page_rows(s["t"], most, s["ln"], s["nn"])), plan)
        torch.cuda.synchronize()
        assert torch.equal(s["o"], want)
        for r in others.values():  # each with a plan of its own
            tadm.tadm_pages_share(m, r, 2, 1, plan)
            attend(m, dict(s, r=r), plan)
        torch.cuda.synchronize()
    finally:
        tadm.tadm_model_destroy(m)
