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
          layer=1, fill=7.0):
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
            worst = max(worst, float((err / bo).max()))
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
