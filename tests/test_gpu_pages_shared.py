"""Attention over pages that rows share, on the GPU, against the float64 oracle.

Groups are compared exactly; attention is held to the bounds of attention over pages (test_gpu_pages): the
parts that a column is joined from add roundings of float32 only, which those bounds count."""
import numpy as np
import pytest
import torch

from oracle import pages as P
from test_gpu_pages import DT, bounds, cap_of, i32, model, random_pages, to_gpu, window

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def tables(rng, prompts, max_pages, spare=2):
    """Tables of rows that share: prompts is a list of (whole pages of the prompt, lengths of its rows)."""
    need = sum(w for w, _ in prompts) + sum(max(0, -(-ln // 64) - w) for w, rows in prompts for ln in rows)
    ids = rng.permutation(need + spare).tolist()
    table, lens = [], []
    for whole, rows in prompts:
        common = [ids.pop() for _ in range(whole)]
        for ln in rows:
            row = common[:-(-ln // 64)]
            row = row + [ids.pop() for _ in range(-(-ln // 64) - len(row))]
            table.append(row + [-1] * (max_pages - len(row)))
            lens.append(ln)
    return np.array(table), lens, need + spare


def scratch(size):
    return torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda")  # NaN: nothing relies on it


def share(m, r, n, min_pages=1):
    data = scratch(tadm.tadm_pages_plan_bytes(m, r, n))
    plan = tadm.page_plan(data)
    plan.keep = data
    lead, pages = i32([-5] * r.B), i32([-5] * r.B)
    tadm.tadm_pages_share(m, r, n, min_pages, plan, lead, pages)
    return plan, lead, pages


def check(dtype, H, Hkv, dh, prompts, news, seed, min_pages=1, windowed=True, want_lse=True, host_lens=False, edit=None,
          layer=1, fill=7.0, seen=None):
    rng = np.random.default_rng(seed)
    mp = max(1, max(-(-ln // 64) for _, rows in prompts for ln in rows))
    table, lens, n_pages = tables(rng, prompts, mp)
    pages = random_pages(rng, n_pages, 2, Hkv, dh)
    if edit:
        edit(table, lens, pages)
    B, n = len(lens), max(max(news), 1)
    cap = cap_of(n)
    q = torch.from_numpy(rng.normal(size=(B, H, n, dh))).to(DT[dtype])
    k, vt = window(rng, B, Hkv, cap, dh, dtype)
    for b in range(B):  # what lies behind a row's window counts for nothing
        k[b, :, news[b]:], vt[b, :, :, news[b]:] = float("nan"), float("nan")
    data, scale, p = to_gpu(pages)
    m = model(dtype, H, Hkv, dh)
    try:
        t, ln, nn = i32(table), i32(lens), i32(news)
        r = tadm.page_rows(t, mp * 64 if not host_lens else lens[0], None if host_lens else ln, nn)
        plan, lead, common = share(m, r, n, min_pages)
        if seen is not None:
            seen.append(plan)
        o = torch.full((B, n, H * dh), fill, dtype=DT[dtype], device="cuda")
        lse = torch.full((B, H, n), fill, device="cuda") if want_lse else None
        work = scratch(tadm.tadm_pages_attend_shared_work(m, r, n))
        qd, kd, vd = q.cuda(), k.cuda() if windowed else None, vt.cuda() if windowed else None
        tadm.tadm_pages_attend_shared(m, p, layer, r, plan, qd, n, kd, vd, cap if windowed else 0, o, lse, work)
        torch.cuda.synchronize()
        ref_lead, ref_common = P.groups(table.tolist(), lens, min_pages)
        assert lead.tolist() == ref_lead and common.tolist() == ref_common
        first = o.clone(), None if lse is None else lse.clone()
        tadm.tadm_pages_attend_shared(m, p, layer, r, plan, qd, n, kd, vd, cap if windowed else 0, o, lse, work)
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.uint8), first[0].view(torch.uint8))  # the same bits in every run
        og, lg = o.double().cpu().numpy().reshape(B, n, H, dh), None if lse is None else lse.double().cpu().numpy()
        worst = 0.0
        for b in range(B):
            nb = news[b]
            assert (og[b, nb:] == fill).all() and (lg is None or (lg[b, :, nb:] == fill).all())
            if nb == 0:
                continue
            pk, pv, there = pages.read(layer, table[b], lens[b])
            pk, pv = pk[:, there], pv[:, there]
            if windowed:
                pk = np.concatenate([pk, k[b, :, :nb].double().numpy()], 1)
                pv = np.concatenate([pv, vt[b, :, :, :nb].double().numpy().transpose(0, 2, 1)], 1)
            qb = q[b, :, :nb].double().numpy()
            ref, ref_lse = P.attend(qb, pk, pv)
            if np.isnan(pk).any() or np.isnan(pv).any():
                seen = np.isnan(ref)
                assert np.array_equal(np.isnan(og[b, :nb]), seen)
                continue
            bo, bl = bounds(dtype, qb, pk, pv)
            err = np.abs(og[b, :nb] - ref)
            worst = max(worst, float((err / np.maximum(bo, 1e-30)).max()))
            assert (err <= bo).all(), (b, float((err / bo).max()))
            if lg is not None:
                same = lg[b, :, :nb] == ref_lse
                with np.errstate(invalid="ignore"):
                    assert (same | (np.abs(lg[b, :, :nb] - ref_lse) <= bl)).all(), b
        print(f"worst error / bound {worst:.3f}")
    finally:
        tadm.tadm_model_destroy(m)


ATTEND = [
    # dtype, H, Hkv, dh, prompts: (whole shared pages, lengths of the rows), new tokens
    ("f32", 4, 4, 16, [(5, [345, 320, 333])], [24, 1, 17]),
    ("f32", 2, 1, 20, [(1, [64, 65]), (0, [0]), (3, [200, 192, 500])], [3, 4, 5, 6, 1, 2]),
    ("f32", 4, 2, 4, [(2, [128, 128]), (2, [130, 150])], [40, 40, 1, 2]),
    ("f32", 2, 2, 128, [(9, [577, 640, 600])], [2, 2, 2]),
    ("bf16", 4, 4, 64, [(3, [192, 200, 255])], [1, 1, 1]),                      # sets of 16 columns
    ("bf16", 4, 2, 64, [(3, [192, 200, 255, 256, 300])], [3, 1, 2, 3, 0]),      # 32
    ("bf16", 4, 2, 64, [(8, [512, 513, 600])], [10, 9, 8]),                     # 64
    ("bf16", 4, 2, 64, [(8, [512, 513, 600]), (1, [64])], [30, 70, 64, 5]),     # own columns of a block 128, partial sets
    ("bf16", 12, 12, 64, [(15, [1000, 961, 980]), (12, [800, 768, 777, 790])], [1] * 7),
    ("bf16", 4, 4, 128, [(2, [128, 129])], [1, 1]),
    ("bf16", 8, 2, 128, [(20, [1280, 1300, 1400, 1290])], [1, 2, 2, 1]),
    ("bf16", 8, 2, 128, [(20, [1300, 1280, 1400])], [7, 8, 5]),
    ("bf16", 8, 2, 128, [(30, [2000, 1920, 2100])], [64, 60, 33]),
    ("bf16", 4, 1, 128, [(40, [2560] * 33)], [1] * 33),                          # 132 columns: a second tile
    ("bf16", 2, 2, 128, [(70, [4500, 4480])], [130, 200]),                       # many splits
    ("bf16", 4, 2, 128, [(0, [0]), (0, [63]), (0, [700]), (0, [64])], [1, 40, 20, 64]),  # nothing to share
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
@pytest.mark.parametrize("windowed", [True, False])
def test_attention_of_rows_that_share(case, windowed):
    dtype, H, Hkv, dh, prompts, news = ATTEND[case]
    check(dtype, H, Hkv, dh, prompts, news, 100 + case, windowed=windowed)


def spread(length, rows, step=7):
    return [length + step * i for i in range(rows)]


# Calls large enough that the plan attends to shared pages together: sets of 16, 32, 64 and 128 columns, several tiles of them,
# several groups with rows between that share nothing, heads shared out over a block's waves, splits on both sides.
TOGETHER = [
    # dtype, H, Hkv, dh, prompts, new tokens
    ("f32", 4, 4, 16, [(60, spread(3840, 16))], [1] * 16),
    ("f32", 4, 2, 20, [(60, spread(3845, 20)), (0, [100, 0]), (50, spread(3200, 14))], [2, 1] * 18),
    ("bf16", 16, 16, 128, [(30, spread(1930, 9))], [1] * 9),
    ("bf16", 16, 16, 64, [(40, spread(2560, 24))], [1] * 24),
    ("bf16", 16, 8, 128, [(40, spread(2561, 18))], [1, 2] * 9),
    ("bf16", 8, 8, 64, [(64, spread(4096, 40, 3))], [3, 4] * 20),
    ("bf16", 32, 16, 128, [(20, spread(1280, 64, 9))], [1] * 64),
    ("bf16", 16, 16, 128, [(30, spread(1950, 10)), (0, [70, 3]), (33, spread(2150, 20)), (0, [0])], [1, 1, 0] * 11),
    ("bf16", 16, 16, 128, [(30, spread(1921, 35)), (29, spread(1900, 35))], [1] * 70),  # more rows than a wave
]


def shared_work(plan):
    """Items of a plan on shared pages: those without a window."""
    words = plan.keep.cpu().numpy()[:plan.bytes // 4 * 4].view(np.int32)
    items = words[16 + 8 * plan.B:][:12 * words[0]].reshape(-1, 12)
    return int((items[:, 9] == 0).sum()), items


@pytest.mark.parametrize("case", range(len(TOGETHER)))
@pytest.mark.parametrize("windowed", [True, False])
def test_attention_over_shared_pages(case, windowed):
    dtype, H, Hkv, dh, prompts, news = TOGETHER[case]
    plans = []
    check(dtype, H, Hkv, dh, prompts, news, 300 + case, windowed=windowed, seen=plans)
    assert shared_work(plans[0])[0] > 0


def test_plans_of_other_groups():
    """min_pages parts rows that share fewer; the same rows, lengths given by the host, without a window, without lse."""
    prompts = [(3, spread(192, 4)), (12, spread(768, 5)), (1, [70, 64])]
    for least in (1, 2, 4, 13, 1000):
        check("bf16", 4, 4, 64, prompts, [2] * 11, 5, min_pages=least)
    check("bf16", 4, 4, 64, [(7, [448] * 6)], [2] * 6, 6, host_lens=True)
    check("bf16", 16, 16, 128, [(30, spread(1930, 9))], [1] * 9, 7, want_lse=False)


@pytest.mark.parametrize("page", [0, 1, 29])
def test_absent_and_nan_pages(page):
    def absent(table, lens, pages):
        table[:, page] = -1
        table[4:, 17] = pages.n_pages  # some rows of the group only: it shares what comes before

    check("bf16", 16, 16, 128, [(30, spread(1930, 12))], [1] * 12, 11, edit=absent)

    def nan(table, lens, pages):
        pages.codes[table[0, page], :, 3, 0, 5] = 0x7f
        pages.codes[table[0, page], :, 5, 1, 70] = 0xff

    check("bf16", 16, 16, 128, [(30, spread(1930, 12))], [1] * 12, 12, edit=nan)


def test_the_most_rows():
    """1 024 rows in groups of one to forty."""
    rng = np.random.default_rng(13)
    prompts, left = [], 1024
    while left:
        rows = min(left, int(rng.integers(1, 41)))
        whole = int(rng.integers(0, 5))
        prompts.append((whole, rng.integers(64 * whole, 64 * whole + 90, size=rows).tolist()))
        left -= rows
    check("f32", 2, 1, 8, prompts, rng.integers(0, 3, size=1024).tolist(), 13)


def test_long_prompts_are_searched_whole():
    """More pages than the plan compares at once, parting late: 64 rows of 300 pages, of which neighbours part at any page."""
    rng = np.random.default_rng(14)

    def part(table, lens, pages):
        for b in range(1, 64):
            table[b, int(rng.integers(1, 300)):300] = pages.n_pages + b  # absent, and another id for each row

    check("f32", 1, 1, 4, [(300, [300 * 64 + b for b in range(64)])], [1] * 64, 14, edit=part)


def state_of(m, rng, dtype, H, Hkv, dh, prompts, n):
    mp = max(-(-ln // 64) for _, rows in prompts for ln in rows) + 1
    table, lens, n_pages = tables(rng, prompts, mp)
    data, scale, p = to_gpu(random_pages(rng, n_pages, 1, Hkv, dh))
    B, cap = len(lens), cap_of(n)
    k, vt = window(rng, B, Hkv, cap, dh, dtype)
    s = dict(data=data, scale=scale, p=p, t=i32(table), ln=i32(lens), nn=i32([n] * B), n=n, cap=cap, k=k.cuda(), vt=vt.cuda(),
             q=torch.from_numpy(rng.normal(size=(B, H, n, dh))).to(DT[dtype]).cuda(), mp=mp, table=table, lens=lens,
             o=torch.zeros(B, n, H * dh, dtype=DT[dtype], device="cuda"), lse=torch.zeros(B, H, n, device="cuda"))
    s["r"] = tadm.page_rows(s["t"], mp * 64, s["ln"], s["nn"])
    s["work"] = scratch(tadm.tadm_pages_attend_shared_work(m, s["r"], n))
    return s


def attend(m, s, plan, o=None, lse=None, work=None):
    tadm.tadm_pages_attend_shared(m, s["p"], 0, s["r"], plan, s["q"], s["n"], s["k"], s["vt"], s["cap"], s["o"] if o is None else o,
                                  s["lse"] if lse is None else lse, s["work"] if work is None else work)


@pytest.mark.parametrize("dtype, H, Hkv, dh, prompts, n", [
    ("bf16", 16, 16, 128, [(30, spread(1930, 12))], 1),
    ("f32", 4, 4, 16, [(60, spread(3840, 16))], 2),
])
def test_captured_passes_follow_tables_and_lengths(dtype, H, Hkv, dh, prompts, n):
    """A captured plan with the call that takes it, replayed over other tables and lengths, equals the eager calls."""
    rng = np.random.default_rng(15)
    m = model(dtype, H, Hkv, dh)
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    try:
        s = state_of(m, rng, dtype, H, Hkv, dh, prompts, n)
        data = scratch(tadm.tadm_pages_plan_bytes(m, s["r"], n))
        plan = tadm.page_plan(data)
        side.wait_stream(main)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            tadm.tadm_set_stream(m, side.cuda_stream)
            with torch.cuda.graph(graph, stream=side):
                tadm.tadm_pages_share(m, s["r"], n, 1, plan)
                attend(m, s, plan)
            tadm.tadm_set_stream(m, main.cuda_stream)
        main.wait_stream(side)
        B = len(s["lens"])
        for change in range(5):
            table, lens = s["table"].copy(), np.array(s["lens"])
            if change == 1:
                lens -= 64 * np.arange(B)  # fewer whole pages in common
            if change == 2:
                table[B // 2:, 3] = table[:B - B // 2, -2]  # another page in half of the rows
            if change == 3:
                lens[:] = 5
            s["t"].copy_(i32(table))
            s["ln"].copy_(i32(lens))
            s["o"].zero_()
            graph.replay()
            torch.cuda.synchronize()
            other, _, _ = share(m, s["r"], n)
            o, lse = torch.zeros_like(s["o"]), torch.zeros_like(s["lse"])
            attend(m, s, other, o, lse)
            torch.cuda.synchronize()
            assert torch.equal(s["o"], o) and torch.equal(s["lse"], lse), change
    finally:
        tadm.tadm_set_stream(m, main.cuda_stream)
        tadm.tadm_model_destroy(m)


def test_calls_that_overlap_on_one_plan():
    rng = np.random.default_rng(16)
    m = model("bf16", 16, 16, 128)
    main, streams = torch.cuda.current_stream(), [torch.cuda.Stream() for _ in range(2)]
    try:
        s = state_of(m, rng, "bf16", 16, 16, 128, [(30, spread(1930, 12))], 1)
        plan, _, _ = share(m, s["r"], 1)
        attend(m, s, plan)
        torch.cuda.synchronize()
        outs = [(torch.zeros_like(s["o"]), torch.zeros_like(s["lse"]), torch.empty_like(s["work"])) for _ in streams]
        torch.cuda.synchronize()
        for _ in range(20):
            for st, (o, lse, work) in zip(streams, outs):
                tadm.tadm_set_stream(m, st.cuda_stream)
                attend(m, s, plan, o, lse, work)
        torch.cuda.synchronize()
        for o, lse, _ in outs:
            assert torch.equal(o, s["o"]) and torch.equal(lse, s["lse"])
    finally:
        tadm.tadm_set_stream(m, main.cuda_stream)
        tadm.tadm_model_destroy(m)


def test_refusals_of_plans_and_scratch():
    rng = np.random.default_rng(17)
    m, other = model("bf16", 4, 4, 64), model("bf16", 8, 4, 64)
    try:
        s = state_of(m, rng, "bf16", 4, 4, 64, [(3, [192, 200])], 2)
        plan, _, _ = share(m, s["r"], 2)
        with pytest.raises(tadm.TadmError) as e:  # a plan that no call has laid out
            attend(m, s, tadm.page_plan(plan.keep))
        assert e.value.status == tadm.TADM_ERR_STATE
        for field, value in (("n", 1), ("B", 1), ("len", 64), ("max_pages", 2), ("n_heads", 8), ("n_kv_heads", 2), ("dtype", 0)):
            wrong = tadm.tadm_page_plan.from_buffer_copy(plan)
            setattr(wrong, field, value)
            with pytest.raises(tadm.TadmError) as e:
                attend(m, s, wrong)
            assert e.value.status == tadm.TADM_ERR_STATE and "plan" in str(e.value)
        with pytest.raises(tadm.TadmError) as e:  # a model of other heads
            attend(other, s, plan)
        assert e.value.status == tadm.TADM_ERR_STATE
        for work in (None, s["work"][:-16], s["work"][8:]):
            with pytest.raises(tadm.TadmError, match="scratch"):
                tadm.tadm_pages_attend_shared(m, s["p"], 0, s["r"], plan, s["q"], 2, s["k"], s["vt"], s["cap"], s["o"], s["lse"], work)
        size = tadm.tadm_pages_plan_bytes(m, s["r"], 2)
        with pytest.raises(tadm.TadmError, match="plan of"):
            tadm.tadm_pages_share(m, s["r"], 2, 1, tadm.page_plan(scratch(size)[:size - 16]))
        with pytest.raises(tadm.TadmError, match="aligned"):
            tadm.tadm_pages_share(m, s["r"], 2, 1, tadm.page_plan(scratch(size + 16)[4:]))
        attend(m, s, plan)
        torch.cuda.synchronize()
    finally:
        tadm.tadm_model_destroy(m)
        tadm.tadm_model_destroy(other)
