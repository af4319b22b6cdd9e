"""Attention by plans that do not fit the call, on the GPU: tables and lengths that changed after the plan was made, and
memory that no plan has been laid out in yet (a capture records the plan, a replay makes it).  The results are
void then; nothing around them is touched, and a plan made anew gives the same bits as before."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DT, cap_of, i32, model, random_pages, to_gpu, window
from test_gpu_pages_shared import spread, tables

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

GUARD = 4096  # bytes on either side


class Guarded:
    """A tensor of `size` bytes with others before and behind it in the same allocation."""

    def __init__(self, size, fill):
        self.all = torch.full((size + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        self.bytes = self.all[GUARD:GUARD + size]
        self.bytes.fill_(fill)

    def intact(self):
        return bool((self.all[:GUARD] == 0xA5).all() and (self.all[-GUARD:] == 0xA5).all())


class Call:
    def __init__(self, dtype, H, Hkv, dh, prompts, n, fill):
        rng = np.random.default_rng(3)
        self.m, self.n = model(dtype, H, Hkv, dh), n
        self.mp = max(-(-ln // 64) for _, rows in prompts for ln in rows)
        table, lens, n_pages = tables(rng, prompts, self.mp)
        self.data, self.scale, self.p = to_gpu(random_pages(rng, n_pages, 1, Hkv, dh))
        B, self.cap = len(lens), cap_of(n)
        self.t, self.ln, self.nn = i32(table), i32(lens), i32([n] * B)
        self.rows = tadm.page_rows(self.t, self.mp * 64, self.ln, self.nn)
        k, vt = window(rng, B, Hkv, self.cap, dh, dtype)
        self.k, self.vt = k.cuda(), vt.cuda()
        self.q = torch.from_numpy(rng.normal(size=(B, H, n, dh))).to(DT[dtype]).cuda()
        width = 4 if dtype == "f32" else 2
        self.mem = dict(plan=Guarded(tadm.tadm_pages_plan_bytes(self.m, self.rows, n), fill),
                        work=Guarded(tadm.tadm_pages_attend_shared_work(self.m, self.rows, n), 0xff),
                        o=Guarded(B * n * H * dh * width, 0), lse=Guarded(B * H * n * 4, 0),
                        lead=Guarded(B * 4, 0), pages=Guarded(B * 4, 0))
        self.o = self.mem["o"].bytes.view(DT[dtype]).view(B, n, H * dh)
        self.lse = self.mem["lse"].bytes.view(torch.float32).view(B, H, n)
        self.plan = tadm.page_plan(self.mem["plan"].bytes)

    def share(self):
        tadm.tadm_pages_share(self.m, self.rows, self.n, 1, self.plan, self.mem["lead"].bytes.view(torch.int32),
                              self.mem["pages"].bytes.view(torch.int32))

    def attend(self, plan=None):
        tadm.tadm_pages_attend_shared(self.m, self.p, 0, self.rows, plan or self.plan, self.q, self.n, self.k, self.vt, self.cap,
                                      self.o, self.lse, self.mem["work"].bytes)
        torch.cuda.synchronize()
        for name, g in self.mem.items():
            assert g.intact(), name

    def fresh(self):
        """(o, lse) by a plan of the tables and lengths as they are."""
        self.share()
        self.o.zero_(), self.lse.zero_()
        self.attend()
        return self.o.clone(), self.lse.clone()


CALLS = [
    ("f32", 4, 2, 16, [(60, spread(3845, 20)), (0, [100, 0]), (50, spread(3200, 14))], 2),
    ("bf16", 16, 16, 64, [(40, spread(2560, 24))], 1),
    ("bf16", 32, 16, 128, [(20, spread(1280, 64, 9))], 1),
    ("bf16", 8, 8, 64, [(64, spread(4096, 40, 3))], 4),
    ("bf16", 4, 2, 128, [(8, [512, 513, 600]), (1, [64])], 70),
]


@pytest.mark.parametrize("case", range(len(CALLS)))
def test_plans_of_other_tables_and_lengths(case):
    c = Call(*CALLS[case], fill=0xff)
    try:
        B, most = c.t.shape[0], c.mp * 64
        rng = np.random.default_rng(case)
        table, lens = c.t.clone(), c.ln.clone()
        want = c.fresh()
        for ln, nn in ((torch.zeros_like(lens), None), (torch.full_like(lens, most), None), (i32(rng.integers(0, most + 1, size=B)), None),
                       (lens, i32(rng.integers(0, c.n + 1, size=B))), (lens, torch.zeros_like(lens)), (lens.flip(0), None)):
            c.t.copy_(table), c.ln.copy_(lens), c.nn.fill_(c.n)
            c.share()
            c.ln.copy_(ln)
            if nn is not None:
                c.nn.copy_(nn)
            c.attend()
            c.share()  # and the other way: a plan of the changed ones over those before
            c.ln.copy_(lens), c.nn.fill_(c.n)
            c.attend()
        for other in (torch.full_like(table, -1), torch.full_like(table, 2 ** 31 - 1), table.flip(0)):
            c.share()
            c.t.copy_(other)
            c.attend()
            c.t.copy_(table)
        assert all(torch.equal(a, b) for a, b in zip(c.fresh(), want))
    finally:
        tadm.tadm_model_destroy(c.m)


@pytest.mark.parametrize("case", range(len(CALLS)))
@pytest.mark.parametrize("fill", [0, 0xff, 0x7f, 0x01])
def test_a_captured_plan_before_its_first_replay(case, fill):
    """The capture fills the descriptor and lays out nothing; an eager call by it finds the memory as it was."""
    c = Call(*CALLS[case], fill=fill)
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    try:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            tadm.tadm_set_stream(c.m, side.cuda_stream)
            with torch.cuda.graph(graph, stream=side):
                c.share()
            tadm.tadm_set_stream(c.m, main.cuda_stream)
        torch.cuda.synchronize()
        assert (c.mem["plan"].bytes == fill).all()
        c.attend()
        assert (c.o == 0).all() and (c.lse == 0).all()  # no such words are an item or a row's parts
        for _ in range(2):
            c.mem["plan"].bytes.fill_(fill)
            graph.replay()
            c.o.zero_(), c.lse.zero_()
            c.attend()
            got = c.o.clone(), c.lse.clone()
            assert all(torch.equal(a, b) for a, b in zip(c.fresh(), got))
    finally:
        tadm.tadm_set_stream(c.m, main.cuda_stream)
        tadm.tadm_model_destroy(c.m)
