"""What lies beside the arrays of the operators for samples of one prompt, and the finite values beside NaN, on the GPU.

Every array is a slice of a larger one, whose bytes on either side stay as they were."""
import numpy as np
import pytest
import torch

import synth
from oracle import draw as D
from oracle import pages as P
from test_gpu_pages import bounds, cap_of, i32, model, random_pages, to_gpu, window
from test_gpu_pages_shared import spread, tables

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

SIDE, MARK = 1024, 0x5A


class Guards:
    def __init__(self):
        self.all = []

    def array(self, values=None, shape=None, dtype=torch.uint8, fill=0xff):
        """A tensor of these values (or bytes of `fill`) inside a larger allocation."""
        if values is not None:
            values = torch.as_tensor(values)
            shape, dtype = tuple(values.shape), values.dtype
        size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        whole = torch.full((size + 2 * SIDE,), MARK, dtype=torch.uint8, device="cuda")
        self.all.append(whole)
        inner = whole[SIDE:SIDE + size]
        inner.fill_(fill)
        t = inner.view(dtype).view(shape)
        if values is not None:
            t.copy_(values)
        return t

    def check(self):
        torch.cuda.synchronize()
        for i, w in enumerate(self.all):
            assert (w[:SIDE] == MARK).all() and (w[-SIDE:] == MARK).all(), i


def word(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32)


@pytest.fixture(scope="module")
def tiny():
    m = tadm.tadm_model_create(tadm.make_config(synth.get_config("tiny"), max_batch=4, max_seq=256))
    tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
    yield m
    tadm.tadm_model_destroy(m)


@pytest.mark.parametrize("rows", [2, 9, 300])
def test_pages_that_come_back_more_often_than_there_are(tiny, rows):
    """A full stack to which every row gives the same two pages: nothing is written behind its last entry."""
    g = Guards()
    ids, state, table = g.array(word([3, 2, 1, 0])), g.array(word([4, 0, 0, 0])), g.array(word([[1, 2]] * rows))
    stack = tadm.page_stack(ids, state)
    tadm.tadm_pages_release(tiny, stack, tadm.page_rows(table, 0, i32([0] * rows), i32([128] * rows)), 128)
    g.check()
    assert ids.tolist() == [3, 2, 1, 0] and state.tolist() == [4, 0, 0, 0] and table.eq(-1).all()
    # from three pages on there is room for one of them
    state.copy_(word([3, 0, 0, 0])), table.copy_(word([[1, 2]] * rows))
    tadm.tadm_pages_release(tiny, stack, tadm.page_rows(table, 0, i32([0] * rows), i32([128] * rows)), 128)
    g.check()
    assert ids.tolist() == [3, 2, 1, 1] and state.tolist() == [4, 0, 0, 0] and table.eq(-1).all()


@pytest.mark.parametrize("lens, news, free", [
    ([0], [1], 1), ([63, 64, 65, 0], [1, 1, 1, 1], 4), ([100, 7, 333, 64], [64, 500, 1, 128], 5), ([0, 1, 64, 4000], [4096, 2047, 2049, 6000], 300),
    ([128] * 300, [1] * 300, 299), ([5] * 4096, [60] * 4096, 4000),
])
def test_tables_and_stacks(tiny, lens, news, free):
    rng, g = np.random.default_rng(free), Guards()
    B, n = len(lens), max(news)
    mp = max(P._up(a + b) for a, b in zip(lens, news))
    size = sum(P._up(x) for x in lens) + free
    ids = rng.permutation(size).tolist()
    table = [[ids.pop() for _ in range(P._up(x))] + [-1] * (mp - P._up(x)) for x in lens]
    ids += [-7] * (size - free)
    t, s, st = g.array(word(table)), g.array(word(ids)), g.array(word([free, 0, 0, 0]))
    ln, nw, granted = g.array(word(lens)), g.array(word(news)), g.array(shape=(B,), dtype=torch.int32)
    slots = g.array(shape=(B, n), dtype=torch.int64)
    stack, rows = tadm.page_stack(s, st), tadm.page_rows(t, mp * 64, ln, nw)
    ref, ref_slots, left = P.assign(table, lens, news, ids, free, size)
    tadm.tadm_pages_assign(tiny, stack, rows, n, granted, slots)
    g.check()
    assert granted.tolist() == ref and t.tolist() == table and st.tolist() == [left, 0, 0, 0]
    assert slots.tolist() == [x + [-1] * (n - len(x)) for x in ref_slots]
    left = P.release(table, lens, ref, ids, left, size)
    tadm.tadm_pages_release(tiny, stack, tadm.page_rows(t, mp * 64, ln, granted), n)
    g.check()
    assert t.tolist() == table and st.tolist() == [left, 0, 0, 0] and s[:left].tolist() == ids[:left]
    assert ln.tolist() == lens and nw.tolist() == news


@pytest.mark.parametrize("R, V", [(1, 262144), (3, 16385), (9, 128256), (5, 1), (1030, 700)])
@pytest.mark.parametrize("sd", [2.0, 0.05])
def test_draws(R, V, sd):
    """Rows in several blocks and in one, with lists that hold their entries and ones that overflow."""
    rng, g = np.random.default_rng(R + V), Guards()
    m = tadm.tadm_model_create(tadm.make_config(synth.get_config("tiny", vocab=V), max_batch=1, max_seq=64))
    tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
    try:
        rows, u = (rng.normal(size=(R, V)) * sd).astype(np.float32), rng.random(R).astype(np.float32)
        s = dict(temperature=rng.choice([0.0, 0.7, 1.0], size=R).astype(np.float32), top_k=rng.choice([0, 1, 50, V // 2 + 1], size=R).astype(np.int32),
                 top_p=rng.choice([1.0, 0.9, 0.5], size=R).astype(np.float32), min_p=rng.choice([0.0, 0.05], size=R).astype(np.float32))
        logits = g.array(rows)
        dev = {k: g.array(v) for k, v in s.items()}
        ud, token, logp = g.array(u), g.array(shape=(R,), dtype=torch.int32), g.array(shape=(R,), dtype=torch.float32)
        work = g.array(shape=(tadm.tadm_sample_rows_work(m, R),))
        tadm.tadm_sample_rows(m, logits, tadm.row_settings(**dev), ud, token, logp, work if work.numel() else None)
        g.check()
        assert token.tolist() == [D.draw(rows[r], u[r], **{k: v[r] for k, v in s.items()})[0] for r in range(R)]
    finally:
        tadm.tadm_model_destroy(m)


@pytest.mark.parametrize("page", [0, 29])
def test_finite_values_beside_nan(page):
    """A NaN key takes the results of its head in the rows that name its page, a NaN value those of its place of the
    head width; all others are what they are without."""
    H = Hkv = 16
    dh, n = 128, 1
    rng, g = np.random.default_rng(12), Guards()
    table, lens, n_pages = tables(rng, [(30, spread(1930, 12)), (0, [100])], 32)
    pages = random_pages(rng, n_pages, 1, Hkv, dh)
    pages.codes[table[0, page], 0, 3, 0, 5] = 0x7f
    pages.codes[table[0, page], 0, 5, 1, 70] = 0xff  # value 70 / 64 of position 70 % 64
    B = len(lens)
    q = torch.from_numpy(rng.normal(size=(B, H, n, dh))).bfloat16()
    k, vt = window(rng, B, Hkv, cap_of(n), dh, "bf16")
    data, scale, p = to_gpu(pages)
    m = model("bf16", H, Hkv, dh)
    try:
        r = tadm.page_rows(i32(table), 32 * 64, i32(lens), i32([n] * B))
        plan = tadm.page_plan(g.array(shape=(tadm.tadm_pages_plan_bytes(m, r, n),)))
        o, lse = g.array(shape=(B, n, H * dh), dtype=torch.bfloat16), g.array(shape=(B, H, n), dtype=torch.float32)
        work = g.array(shape=(tadm.tadm_pages_attend_shared_work(m, r, n),))
        tadm.tadm_pages_share(m, r, n, 1, plan)
        tadm.tadm_pages_attend_shared(m, p, 0, r, plan, q.cuda(), n, k.cuda(), vt.cuda(), cap_of(n), o, lse, work)
        g.check()
        og, lg = o.double().cpu().numpy().reshape(B, n, H, dh), lse.double().cpu().numpy()
        for b in range(B):
            pk, pv, _ = pages.read(0, table[b], lens[b])
            pk = np.concatenate([pk, k[b, :, :n].double().numpy()], 1)
            pv = np.concatenate([pv, vt[b, :, :, :n].double().numpy().transpose(0, 2, 1)], 1)
            qb = q[b].double().numpy()
            ref, ref_lse = P.attend(qb, pk, pv)
            want = np.zeros((n, H, dh), dtype=bool)
            if b < 12:
                want[:, 3], want[:, 5, 70 // 64] = True, True
            assert np.array_equal(np.isnan(ref), want) and np.array_equal(np.isnan(og[b]), want)
            bo, bl = bounds("bf16", qb, np.nan_to_num(pk), np.nan_to_num(pv))
            assert (np.abs(og[b] - ref) <= bo)[~want].all()
            fine = ~np.isnan(ref_lse)
            assert np.array_equal(fine, ~np.isnan(lg[b])) and (np.abs(lg[b] - ref_lse) <= bl)[fine].all()
    finally:
        tadm.tadm_model_destroy(m)
