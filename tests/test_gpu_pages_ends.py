"""The page operators at the ends of their ranges, on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import pages as P

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_pages import DT, bounds, cap_of, i32, model, random_pages, run_attend, to_gpu, window  # noqa: E402
from test_pages_ends import TOPS  # noqa: E402


# ------------------------------------------------------------------ append, read
@pytest.mark.parametrize("dtype, dh", [("f32", 4), ("f32", 20), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("length, n", [(0, 64), (3, 15), (5, 1), (0, 70), (40, 30), (64, 16)])
def test_the_largest_values(dtype, dh, length, n):
    """Codes and scales as the oracle's, and every finite value reads back finite: values up to the largest of the
    type, beside infinities and NaN, into empty pages and behind positions whose scale grows or stays 2^120."""
    Hkv, cap = 2, cap_of(n)
    last = (length + n - 1) // 64 + 1
    pages = P.Pages(np.zeros((4, 1, Hkv, 2, 64 * dh), np.uint8), np.ones((4, 1, Hkv, 2)))
    rng = np.random.default_rng(dh + n)
    x = rng.normal(size=(1, Hkv, cap, dh)) * 1e37
    for t, top in enumerate(TOPS):
        x[0, t % Hkv, t * 13 % n, t % dh] = top * (-1) ** t
    x[0, 0, n - 1, 0], x[0, 1, n // 2, 1], x[0, 1, 0, 2] = np.inf, -np.inf, np.nan
    most = torch.finfo(DT[dtype]).max
    k = torch.from_numpy(np.where(np.isfinite(x), np.clip(x, -most, most), x)).to(DT[dtype])
    v = torch.flip(k, (1,))
    data, scale, p = to_gpu(pages)
    m = model(dtype, Hkv, Hkv, dh)
    try:
        t = i32([[2, 0, 3]])
        steps = [(0, k[:, :, :length], v[:, :, :length])] if length else []  # as many of the same values before
        steps.append((length, k[:, :, :n], v[:, :, :n]))
        for at, a, b in steps:
            new, c = a.shape[2], cap_of(a.shape[2])
            kd, vd = torch.zeros(1, Hkv, c, dh, dtype=DT[dtype]), torch.zeros(1, Hkv, dh, c, dtype=DT[dtype])
            kd[:, :, :new], vd[..., :new] = a, b.transpose(2, 3)
            kd, vd = kd.cuda(), vd.cuda()
            tadm.tadm_pages_append(m, p, 0, tadm.page_rows(t, at), kd, vd, new, c)
            pages.append(0, [2, 0, 3], at, a[0].double().numpy(), b[0].double().numpy())
        assert np.array_equal(scale.cpu().double().numpy(), pages.scales)
        got, ref = data.cpu().numpy(), pages.codes
        both_nan = ((got & 0x7f) == 0x7f) & ((ref & 0x7f) == 0x7f)
        assert np.array_equal(np.where(both_nan, 0, got), np.where(both_nan, 0, ref))
        c = 64 * last
        k2, v2 = torch.zeros(1, Hkv, c, dh, dtype=DT[dtype], device="cuda"), torch.zeros(1, Hkv, dh, c, dtype=DT[dtype], device="cuda")
        tadm.tadm_pages_read(m, p, 0, tadm.page_rows(t, length + n), k2, v2, c)
        for side, new in ((k2, k), (v2.transpose(2, 3), v)):
            back = side[:, :, length:length + n].cpu()
            assert torch.equal(back.isfinite(), new[:, :, :n].isfinite()) and not back.isinf().any()
    finally:
        tadm.tadm_model_destroy(m)


# ------------------------------------------------------------------ attention
def test_rows_beyond_a_launch():
    """More rows and K/V heads than a launch has threads for are refused by name, before anything is read; at the
    limit of rows fewer heads are not."""
    m = model("bf16", 256, 256, 64)
    few = model("bf16", 4, 2, 64)
    try:
        pages = P.Pages(np.zeros((1, 1, 256, 2, 64 * 64), np.uint8), np.ones((1, 1, 256, 2)))
        data, scale, p = to_gpu(pages)
        t = i32([[0]])
        r = tadm.page_rows(t, 0)
        r.B = 65535
        q = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
        assert tadm.tadm_pages_attend_work(m, r, 1) == 0 and "2^32 threads" in tadm.last_error()
        with pytest.raises(tadm.TadmError, match="2\\^32 threads") as e:
            tadm.tadm_pages_attend(m, p, 0, r, q, 1, None, None, 0, q, None, None)
        assert e.value.status == tadm.TADM_ERR_INVALID
        refused = tadm.last_error()
        r = tadm.page_rows(t, 64)
        r.B = 65535
        assert tadm.tadm_pages_attend_work(few, r, 256) == 0  # 2^26 queries, in more blocks than any card has at once
        assert tadm.last_error() == refused
    finally:
        tadm.tadm_model_destroy(m)
        tadm.tadm_model_destroy(few)


def held_to_oracle(dtype, pages, table, spans, q, k, vt, o, lse, heads):
    """Rows of an attention over layer 0 (a K/V head per query head), in some heads, and what lies behind each window."""
    B, H, n, dh = q.shape
    o, lse = o.double().cpu().numpy().reshape(B, n, H, dh), lse.double().cpu().numpy()
    for b, (length, new) in enumerate(spans):
        assert np.all(o[b, new:] == 7.0) and np.all(lse[b, :, new:] == 7.0), f"row {b}: padding was written"
        for h in heads if new else ():
            K, V, _ = P.Pages(pages.codes[:, :, h:h + 1].copy(), pages.scales[:, :, h:h + 1].copy()).read(0, table[b], length)
            K = np.concatenate([K, k[b, h:h + 1, :new].double().numpy()], axis=1)
            V = np.concatenate([V, vt[b, h:h + 1, :, :new].double().numpy().transpose(0, 2, 1)], axis=1)
            qh = q[b, h:h + 1, :new].double().numpy()
            ref, ref_lse = P.attend(qh, K, V)
            to, tl = bounds(dtype, qh, K, V)
            assert np.all(np.abs(o[b, :new, h:h + 1] - ref) <= to), (b, h)
            assert np.all(np.abs(lse[b, h, :new] - ref_lse[0]) <= tl[0]), (b, h)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B, n", [(24, 33), (18, 64), (10, 100), (9, 160), (16, 192)])
def test_more_blocks_than_compute_units(dh, B, n):
    """One to three rounds of blocks of 64 and of 128 columns, their last columns empty or not, behind pages."""
    rng = np.random.default_rng(B + dh)
    H = Hkv = 16
    spans = [([130, 64, 0, 200, 321][b % 5], [n, 1, n - 1, 0][b % 4]) for b in range(B)]
    mp, cap = 6, cap_of(n)
    pages = random_pages(rng, B * mp, 1, Hkv, dh)
    table = rng.permutation(B * mp).reshape(B, mp)
    q = torch.from_numpy(rng.normal(size=(B, H, n, dh))).to(torch.bfloat16)
    k, vt = window(rng, B, Hkv, cap, dh, "bf16")
    for b, (_, new) in enumerate(spans):
        k[b, :, new:], vt[b, :, :, new:], q[b, :, new:] = float("nan"), float("nan"), float("nan")
    data, scale, p = to_gpu(pages)
    m = model("bf16", H, Hkv, dh)
    try:
        o, lse = run_attend(m, "bf16", p, 0, table, [a for a, _ in spans], [b for _, b in spans], mp * 64, q, k, vt, cap)
    finally:
        tadm.tadm_model_destroy(m)
    held_to_oracle("bf16", pages, table, spans, q, k, vt, o, lse, (0, Hkv - 1))


@pytest.mark.parametrize("dtype, Hkv, dh, spans, n", [
    # bf16: blocks of 128 and of 64 columns, one and several splits
    ("bf16", 8, 128, [(0, 1000), (100, 999), (64, 513), (0, 0), (300, 1), (37, 960), (128, 1000), (1, 640)], 1000),
    ("bf16", 8, 64, [(0, 1000), (100, 999), (64, 513), (0, 0), (300, 1), (37, 960), (128, 1000), (1, 640)], 1000),
    ("bf16", 2, 128, [(0, 520), (200, 577)], 577),
    ("bf16", 2, 64, [(0, 520), (200, 577)], 577),
    ("bf16", 1, 128, [(0, 1536)], 1536),
    ("f32", 2, 16, [(0, 600), (333, 517)], 600),
])
def test_windows_of_a_prompt(dtype, Hkv, dh, spans, n):
    """Windows of many tiles of their own keys, as appending a prompt has them, behind pages and without."""
    rng = np.random.default_rng(n + dh)
    B, mp, cap = len(spans), 6, cap_of(n)
    pages = random_pages(rng, B * mp, 1, Hkv, dh)
    table = rng.permutation(B * mp).reshape(B, mp)
    q = torch.from_numpy(rng.normal(size=(B, Hkv, n, dh))).to(DT[dtype])
    k, vt = window(rng, B, Hkv, cap, dh, dtype)
    for b, (_, new) in enumerate(spans):
        k[b, :, new:], vt[b, :, :, new:], q[b, :, new:] = float("nan"), float("nan"), float("nan")
    data, scale, p = to_gpu(pages)
    m = model(dtype, Hkv, Hkv, dh)
    try:
        o, lse = run_attend(m, dtype, p, 0, table, [a for a, _ in spans], [b for _, b in spans], mp * 64, q, k, vt, cap)
    finally:
        tadm.tadm_model_destroy(m)
    held_to_oracle(dtype, pages, table, spans, q, k, vt, o, lse, sorted({0, Hkv - 1}))


@pytest.mark.parametrize("length, n", [(9000, 70), (8500, 128)])
def test_blocks_of_128_columns_over_many_tiles(length, n):
    """64 elements a key, enough rows for one split: a wave walks more tiles than a batch of 64.  The rows share
    their pages and queries, so all equal the first, which is held to the oracle in two heads."""
    rng = np.random.default_rng(length)
    Hkv, dh, B, mp = 16, 64, 16, -(-length // 64)
    pages = random_pages(rng, mp + 1, 1, Hkv, dh)
    table = np.tile(rng.permutation(mp + 1)[:mp], (B, 1))
    q = torch.from_numpy(rng.normal(size=(1, Hkv, n, dh))).to(torch.bfloat16).expand(B, -1, -1, -1).contiguous()
    data, scale, p = to_gpu(pages)
    m = model("bf16", Hkv, Hkv, dh)
    try:
        o, lse = run_attend(m, "bf16", p, 0, table, [length] * B, [n] * B, length, q, None, None, 64)
    finally:
        tadm.tadm_model_destroy(m)
    assert torch.equal(o, o[:1].expand_as(o)) and torch.equal(lse, lse[:1].expand_as(lse))
    o, lse = o[0].double().cpu().numpy().reshape(n, Hkv, dh), lse[0].double().cpu().numpy()
    for h in (0, Hkv - 1):
        K, V, _ = P.Pages(pages.codes[:, :, h:h + 1].copy(), pages.scales[:, :, h:h + 1].copy()).read(0, table[0], length)
        qh = q[0, h:h + 1].double().numpy()
        ref, ref_lse = P.attend(qh, K, V)
        to, tl = bounds("bf16", qh, K, V)
        assert np.all(np.abs(o[:, h:h + 1] - ref) <= to) and np.all(np.abs(lse[h] - ref_lse[0]) <= tl[0])
