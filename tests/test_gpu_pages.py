"""The page operators on the GPU against the float64 oracle.

Codes, scales, copies and values read back are compared exactly.  Attention is held to
bounds counted from its roundings (bf16 half a step 2^-8, float32 2^-24): a score sums dh
products in float32, the probabilities are rounded to the model type before they meet V, the
result is rounded once."""
import numpy as np
import pytest
import torch

import synth
from oracle import pages as P

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def model(dtype, H, Hkv, dh):
    cfg = synth.get_config("tiny", dtype=dtype, n_heads=H, n_kv_heads=Hkv, head_dim=dh, d_model=64, vocab=64)
    m = tadm.tadm_model_create(tadm.make_config(cfg, max_batch=4, max_seq=256))
    tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
    return m


def random_pages(rng, n_pages, layers, Hkv, dh):
    """Pages of any codes but NaN, scales 2^-8 .. 2^-5."""
    codes = rng.integers(0, 256, size=(n_pages, layers, Hkv, 2, 64 * dh)).astype(np.uint8)
    codes[(codes & 0x7f) == 0x7f] = 0x3a
    scales = 2.0 ** rng.integers(-8, -4, size=(n_pages, layers, Hkv, 2))
    return P.Pages(codes, scales)


def to_gpu(pages):
    data = torch.from_numpy(pages.codes.copy()).cuda()
    scale = torch.from_numpy(pages.scales.astype(np.float32)).cuda()
    return data, scale, tadm.page_set(data, scale)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def window(rng, B, Hkv, cap, dh, dtype, spread=1.0):
    k = torch.from_numpy(rng.normal(size=(B, Hkv, cap, dh)) * spread).to(DT[dtype])
    vt = torch.from_numpy(rng.normal(size=(B, Hkv, dh, cap))).to(DT[dtype])
    return k, vt


def cap_of(n):
    return -(-n // 64) * 64


# ------------------------------------------------------------------ append
APPEND = [
    # dtype, H, Hkv, dh, rows: (length, new tokens), n
    ("f32", 4, 4, 16, [(0, 1)], 1),
    ("f32", 2, 1, 20, [(63, 2), (5, 9), (130, 0)], 9),
    ("f32", 2, 2, 4, [(1, 200), (64, 64), (0, 200)], 200),
    ("bf16", 4, 2, 64, [(0, 64), (64, 1), (37, 64), (100, 28)], 64),
    ("bf16", 12, 12, 64, [(7, 57), (8, 120), (16, 48)], 130),
    ("bf16", 2, 1, 128, [(31, 129), (0, 3)], 129),
    ("bf16", 8, 2, 128, [(62, 1), (63, 1), (64, 1), (0, 1)], 1),
]


@pytest.mark.parametrize("dtype, H, Hkv, dh, spans, n", APPEND)
@pytest.mark.parametrize("quiet", [False, True])
def test_append_is_exact(dtype, H, Hkv, dh, spans, n, quiet):
    """quiet: new values far below the pages' scales, which then keep them; else they grow."""
    rng = np.random.default_rng(len(spans) + dh + n)
    B, mp = len(spans), max(-(-(a + b) // 64) for a, b in spans) + 1
    pages = random_pages(rng, B * mp + 2, 3, Hkv, dh)
    table = rng.permutation(B * mp + 2)[:B * mp].reshape(B, mp)
    cap = cap_of(n)
    k, vt = window(rng, B, Hkv, cap, dh, dtype, 1e-3 if quiet else 50.0)
    k[0, 0, 0, 0], vt[0, 0, 0, 0] = float("inf"), float("nan")
    k[-1, -1, 0, 1] = -float("inf")
    k[:, :, n:], vt[..., n:] = float("nan"), float("nan")  # columns that no row has
    data, scale, p = to_gpu(pages)
    for b, (length, new) in enumerate(spans):
        pages.append(1, table[b], length, k[b, :, :new].double().numpy(), vt[b, :, :, :new].double().numpy().transpose(0, 2, 1))
    m = model(dtype, H, Hkv, dh)
    try:
        kd, vd, t, ln, nn = k.cuda(), vt.cuda(), i32(table), i32([a for a, _ in spans]), i32([b for _, b in spans])
        r = tadm.page_rows(t, mp * 64, ln, nn)
        tadm.tadm_pages_append(m, p, 1, r, kd, vd, n, cap)
        torch.cuda.synchronize()
        assert np.array_equal(scale.cpu().double().numpy(), pages.scales)
        got, ref = data.cpu().numpy(), pages.codes
        both_nan = ((got & 0x7f) == 0x7f) & ((ref & 0x7f) == 0x7f)
        assert np.array_equal(np.where(both_nan, 0, got), np.where(both_nan, 0, ref))
    finally:
        tadm.tadm_model_destroy(m)


def test_append_rounds_like_the_format():
    """Every midpoint of neighbouring e4m3 values and its float32 neighbours, both signs, at three scales."""
    mid = ((P.POSITIVE[1:] + P.POSITIVE[:-1]) / 2).astype(np.float32)
    x = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(1e9)), P.POSITIVE.astype(np.float32)])
    x = np.concatenate([x, -x, np.zeros(-2 * len(x) % (16 * 64), np.float32)])
    m = model("f32", 1, 1, 16)
    try:
        for e in (-100, 0, 90):
            tiles = (x.astype(np.float64) * 2.0 ** e).reshape(-1, 64, 16)
            tiles[:, 0, 0] = 448.0 * 2.0 ** e  # fixes every page's scale
            n = len(tiles) * 64
            k = torch.from_numpy(tiles.astype(np.float32).reshape(1, 1, n, 16)).cuda()
            vt = k.transpose(2, 3).contiguous()
            pages = P.Pages(np.zeros((len(tiles), 1, 1, 2, 64 * 16), np.uint8), np.ones((len(tiles), 1, 1, 2)))
            data, scale, p = to_gpu(pages)
            t = i32(np.arange(len(tiles))[None])
            tadm.tadm_pages_append(m, p, 0, tadm.page_rows(t, 0), k, vt, n, n)
            torch.cuda.synchronize()
            assert np.all(scale.cpu().numpy() == 2.0 ** e)
            ref = P.encode(tiles / 2.0 ** e)
            got = data.cpu().numpy()[:, 0, 0]
            assert np.array_equal(got[:, 0].reshape(-1, 64, 16), ref)
            assert np.array_equal(got[:, 1].reshape(-1, 16, 64).transpose(0, 2, 1), ref)
    finally:
        tadm.tadm_model_destroy(m)


@pytest.mark.parametrize("top", [0.0, 1e-45, 1e-38, 448.0, 449.0, 3.0e38])
def test_append_scales_at_the_ends(top):
    x = np.zeros((1, 1, 64, 4))
    x[0, 0, 3, 2] = top
    x = x.astype(np.float32)
    pages = P.Pages(np.zeros((1, 1, 1, 2, 256), np.uint8), np.ones((1, 1, 1, 2)))
    data, scale, p = to_gpu(pages)
    pages.append(0, [0], 0, x[0].astype(np.float64), x[0].astype(np.float64))
    m = model("f32", 1, 1, 4)
    try:
        k = torch.from_numpy(x).cuda()
        vt, t = k.transpose(2, 3).contiguous(), i32([[0]])
        tadm.tadm_pages_append(m, p, 0, tadm.page_rows(t, 0), k, vt, 64, 64)
        torch.cuda.synchronize()
        assert np.array_equal(scale.cpu().double().numpy(), pages.scales)
        assert np.array_equal(data.cpu().numpy(), pages.codes)
    finally:
        tadm.tadm_model_destroy(m)


def test_append_keeps_to_the_table_and_to_present_pages():
    """Ids outside the pages and positions behind the table are not written."""
    rng = np.random.default_rng(5)
    pages = random_pages(rng, 6, 1, 2, 16)
    table = np.array([[0, -1, 3], [6, 5, 2147483647]])
    k, vt = window(rng, 2, 2, 192, 16, "f32")
    data, scale, p = to_gpu(pages)
    for b in range(2):
        pages.append(0, table[b], 40, k[b].double().numpy(), vt[b].double().numpy().transpose(0, 2, 1))
    m = model("f32", 2, 2, 16)
    try:
        t, ln, kd, vd = i32(table), i32([40, 40]), k.cuda(), vt.cuda()
        tadm.tadm_pages_append(m, p, 0, tadm.page_rows(t, 192, ln), kd, vd, 192, 192)
        torch.cuda.synchronize()
        assert np.array_equal(data.cpu().numpy(), pages.codes)
        assert np.array_equal(scale.cpu().double().numpy(), pages.scales)
    finally:
        tadm.tadm_model_destroy(m)


# ------------------------------------------------------------------ attention
def bounds(dtype, q, k, v):
    """(bound of o [n, H, dh], bound of lse [H, n]) of the kernel against the oracle."""
    H, n, dh = q.shape
    G, keys = H // k.shape[0], k.shape[1]
    if keys == 0:
        return np.zeros((n, H, dh)), np.zeros((H, n))
    u = 2.0 ** -24
    pv, _ = P.attend(q, k, np.abs(v))  # sum p |v|
    o, lse = P.attend(q, k, v)
    size = np.stack([(np.abs(q[h]) @ np.abs(k[h // G]).T).max(axis=1) for h in range(H)]) / np.sqrt(dh)  # [H, n]
    # a score: dh products summed in any order, its scaling and the reference's subtraction
    ds = ((dh + 8) * size + 8 * (np.abs(lse) + 16)) * u
    # p: the score, the exponential (2 units), its share of sums over the keys and their joins
    dp = 2 * ds + (2 * keys ** 0.5 + 64) * 4 * u
    do = dp.T[:, :, None] * pv
    if dtype == "bf16":
        do = do + 2.0 ** -8 * (pv + np.abs(o))
    else:
        do = do + 4 * u * np.abs(o)
    return do + 1e-30, dp + 4 * u * np.abs(lse)


def run_attend(m, dtype, p, layer, table, lens, news, max_len, q, k, vt, cap, want_lse=True, fill=7.0):
    B, H, n, dh = q.shape
    t, ln, nn = i32(table), i32(lens), i32(news)
    r = tadm.page_rows(t, max_len, ln, nn)
    o = torch.full((B, n, H * dh), fill, dtype=DT[dtype], device="cuda")
    lse = torch.full((B, H, n), fill, device="cuda") if want_lse else None
    size = tadm.tadm_pages_attend_work(m, r, n)
    work = torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda")  # NaN: nothing relies on it
    qd, kd, vd = q.cuda(), None if k is None else k.cuda(), None if vt is None else vt.cuda()
    tadm.tadm_pages_attend(m, p, layer, r, qd, n, kd, vd, cap, o, lse, work)
    torch.cuda.synchronize()
    return o, lse


ATTEND = [
    # dtype, H, Hkv, dh, rows: (length, tokens), n, window keys
    ("f32", 4, 4, 16, [(0, 1)], 1, True),
    ("f32", 4, 4, 16, [(333, 24), (0, 24), (64, 0), (65, 5)], 24, True),
    ("f32", 6, 2, 20, [(100, 7), (1, 1)], 7, True),
    ("f32", 1, 1, 4, [(63, 3), (128, 2), (0, 3)], 3, False),
    ("f32", 2, 1, 100, [(70, 40)], 40, True),
    ("f32", 2, 2, 128, [(190, 17)], 17, False),
    ("bf16", 12, 12, 64, [(777, 1), (64, 1), (0, 1), (1, 1)], 1, True),
    ("bf16", 4, 2, 64, [(129, 100), (500, 63), (0, 77), (63, 0)], 100, True),
    ("bf16", 5, 1, 64, [(200, 13)], 13, True),
    ("bf16", 16, 4, 128, [(200, 1)], 1, True),
    ("bf16", 16, 4, 128, [(1000, 64), (321, 64), (0, 64)], 64, True),
    ("bf16", 16, 16, 128, [(130, 200)], 200, False),
    ("bf16", 4, 2, 128, [(64, 256), (640, 130)], 256, True),
    ("bf16", 32, 1, 128, [(65, 3), (4000, 2)], 3, True),
    ("bf16", 2, 2, 128, [(20000, 1)], 1, True),
    ("bf16", 3, 3, 64, [(9000, 2), (12345, 1)], 2, False),
    # splits of the key axis: float32, two strips of 16 columns, many columns joined by eight groups and by one
    ("f32", 2, 2, 16, [(1500, 20), (3, 1)], 20, True),
    ("bf16", 16, 4, 128, [(3000, 8), (70, 5), (0, 8)], 8, True),
    ("bf16", 4, 4, 64, [(2500, 50)], 50, True),
    ("bf16", 16, 4, 128, [(1300, 200), (64, 1)], 200, True),
]


@pytest.mark.parametrize("dtype, H, Hkv, dh, spans, n, own_keys", ATTEND)
@pytest.mark.parametrize("garbage", [False, True])
def test_attention(dtype, H, Hkv, dh, spans, n, own_keys, garbage):
    """garbage: NaN in every place that no query may see (behind lengths, on pages of nobody, in padding), an
    absent page in each long row."""
    rng = np.random.default_rng(H * dh + n)
    B, mp = len(spans), max(1, max(-(-a // 64) for a, _ in spans)) + 1
    pages = random_pages(rng, B * mp + 1, 2, Hkv, dh)
    table = rng.permutation(B * mp + 1)[:B * mp].reshape(B, mp)
    cap = cap_of(n)
    q = torch.from_numpy(rng.normal(size=(B, H, n, dh))).to(DT[dtype])
    k, vt = window(rng, B, Hkv, cap, dh, dtype)
    if garbage:
        table[:, mp // 2] = [-1, B * mp + 1, 2 ** 31 - 1, -2 ** 31][:B]
        used = np.zeros((pages.n_pages, 64), bool)
        for b, (length, _) in enumerate(spans):
            for i in range(-(-length // 64)):
                if 0 <= table[b, i] < pages.n_pages:
                    used[table[b, i], :min(64, length - 64 * i)] = True
        codes = pages.codes[:, 1]
        keys = codes[:, :, 0].reshape(pages.n_pages, Hkv, 64, dh)
        vals = codes[:, :, 1].reshape(pages.n_pages, Hkv, dh, 64)
        keys[~used[:, None, :].repeat(Hkv, 1)] = 0x7f
        vals.transpose(0, 1, 3, 2)[~used[:, None, :].repeat(Hkv, 1)] = 0xff
        codes[:, :, 0], codes[:, :, 1] = keys.reshape(pages.n_pages, Hkv, -1), vals.reshape(pages.n_pages, Hkv, -1)
        for b, (_, new) in enumerate(spans):
            k[b, :, new:], vt[b, :, :, new:], q[b, :, new:] = float("nan"), float("nan"), float("nan")
    data, scale, p = to_gpu(pages)
    m = model(dtype, H, Hkv, dh)
    try:
        o, lse = run_attend(m, dtype, p, 1, table, [a for a, _ in spans], [b for _, b in spans], mp * 64, q,
                            k if own_keys else None, vt if own_keys else None, cap)
    finally:
        tadm.tadm_model_destroy(m)
    o, lse = o.double().cpu().numpy().reshape(B, n, H, dh), lse.double().cpu().numpy()
    for b, (length, new) in enumerate(spans):
        assert np.all(o[b, new:] == 7.0) and np.all(lse[b, :, new:] == 7.0), f"row {b}: padding was written"
        if new == 0:
            continue
        K, V, there = pages.read(1, table[b], length)
        K, V = K[:, there], V[:, there]
        if own_keys:
            K = np.concatenate([K, k[b, :, :new].double().numpy()], axis=1)
            V = np.concatenate([V, vt[b, :, :, :new].double().numpy().transpose(0, 2, 1)], axis=1)
        qb = q[b, :, :new].double().numpy()
        ref, ref_lse = P.attend(qb, K, V)
        to, tl = bounds(dtype, qb, K, V)
        err = np.abs(o[b, :new] - ref)
        print(f"[pages] row {b}: max err {err.max():.3g}, largest share of its bound {(err / (to + 1e-300)).max():.3g}", flush=True)
        assert np.all(err <= to)
        if K.shape[1] == 0:
            assert np.all(np.isneginf(lse[b, :, :new]))
        else:
            print(f"[pages] row {b}: lse max err {np.abs(lse[b, :, :new] - ref_lse).max():.3g}, largest share of its bound "
                  f"{(np.abs(lse[b, :, :new] - ref_lse) / tl).max():.3g}", flush=True)
            assert np.all(np.abs(lse[b, :, :new] - ref_lse) <= tl)


@pytest.mark.parametrize("Hkv, dh, n, length", [(16, 64, 1, 33100), (16, 64, 40, 9000), (16, 128, 70, 8300)])
def test_attention_of_many_tiles_a_wave(Hkv, dh, n, length):
    """Enough rows that the key axis is not split: a wave walks more tiles than a batch of 64.  The rows share
    their pages and queries, so all equal the first, which is held to the oracle in two heads."""
    rng = np.random.default_rng(length)
    B, mp = 256 // Hkv, -(-length // 64)
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
    o = o[0].double().cpu().numpy().reshape(n, Hkv, dh)
    for h in (0, Hkv - 1):
        one = P.Pages(pages.codes[:, :, h:h + 1].copy(), pages.scales[:, :, h:h + 1].copy())
        K, V, _ = one.read(0, table[0], length)
        qh = q[0, h:h + 1].double().numpy()
        ref, ref_lse = P.attend(qh, K, V)
        to, tl = bounds("bf16", qh, K, V)
        assert np.all(np.abs(o[:, h:h + 1] - ref) <= to)
        assert np.all(np.abs(lse[0, h].double().cpu().numpy() - ref_lse[0]) <= tl[0])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("paged", [True, False])
def test_windows_of_several_tiles_in_full_blocks(dh, paged):
    """Enough columns for blocks of 128: windows of none to three tiles, NaN behind their ends, behind odd and even
    numbers of pages, and alone."""
    rng = np.random.default_rng(dh)
    H = Hkv = 16
    spans = [(0, 130), (1, 64), (64, 65), (65, 1), (128, 128), (150, 0), (70, 129), (300, 100)]
    if not paged:
        spans = [(0, new) for _, new in spans]
    B, n, mp, cap = len(spans), 130, 5, cap_of(130)
    pages = random_pages(rng, B * mp, 1, Hkv, dh)
    table = rng.permutation(B * mp).reshape(B, mp)
    q = torch.from_numpy(rng.normal(size=(B, H, n, dh))).to(torch.bfloat16)
    k, vt = window(rng, B, Hkv, cap, dh, "bf16")
    for b, (_, new) in enumerate(spans):
        k[b, :, new:], vt[b, :, :, new:], q[b, :, new:] = float("nan"), float("nan"), float("nan")
    data, scale, p = to_gpu(pages)
    m = model("bf16", H, Hkv, dh)
    try:
        o, lse = run_attend(m, "bf16", p, 0, table, [a for a, _ in spans], [b for _, b in spans],
                            mp * 64 if paged else 0, q, k, vt, cap)
    finally:
        tadm.tadm_model_destroy(m)
    o, lse = o.double().cpu().numpy().reshape(B, n, H, dh), lse.double().cpu().numpy()
    for b, (length, new) in enumerate(spans):
        assert np.all(o[b, new:] == 7.0) and np.all(lse[b, :, new:] == 7.0), f"row {b}: padding was written"
        for h in (0, Hkv - 1) if new else ():
            K, V, _ = P.Pages(pages.codes[:, :, h:h + 1].copy(), pages.scales[:, :, h:h + 1].copy()).read(0, table[b], length)
            K = np.concatenate([K, k[b, h:h + 1, :new].double().numpy()], axis=1)
            V = np.concatenate([V, vt[b, h:h + 1, :, :new].double().numpy().transpose(0, 2, 1)], axis=1)
            qh = q[b, h:h + 1, :new].double().numpy()
            ref, ref_lse = P.attend(qh, K, V)
            to, tl = bounds("bf16", qh, K, V)
            assert np.all(np.abs(o[b, :new, h:h + 1] - ref) <= to), (b, h)
            assert np.all(np.abs(lse[b, h, :new] - ref_lse[0]) <= tl[0]), (b, h)


def test_overlapping_graphs_with_scratch_of_their_own():
    """Two captured calls replayed at once on two streams, each with its own scratch, equal the eager ones."""
    rng = np.random.default_rng(8)
    H, Hkv, dh, B, mp = 16, 4, 128, 1, 130
    pages = random_pages(rng, mp, 1, Hkv, dh)
    data, scale, p = to_gpu(pages)
    m = model("bf16", H, Hkv, dh)
    try:
        t = i32(rng.permutation(mp)[None])
        runs = []
        for i, length in enumerate((8000, 5001)):
            r = tadm.page_rows(t, length)
            q = torch.randn(B, H, 1, dh, device="cuda").bfloat16()
            size = tadm.tadm_pages_attend_work(m, r, 1)
            assert size > 0
            runs.append(dict(r=r, q=q, o=torch.zeros(B, 1, H * dh, dtype=torch.bfloat16, device="cuda"),
                             work=torch.empty(size, dtype=torch.uint8, device="cuda"), s=torch.cuda.Stream()))

        def call(x):
            tadm.tadm_pages_attend(m, p, 0, x["r"], x["q"], 1, None, None, 0, x["o"], None, x["work"])

        for x in runs:
            call(x)
        torch.cuda.synchronize()
        want = [x["o"].clone() for x in runs]
        for x in runs:
            x["g"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(x["g"], stream=x["s"]):
                tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
                call(x)
        for _ in range(5):
            for x in runs:
                x["o"].zero_()
            torch.cuda.synchronize()
            for x in runs:
                with torch.cuda.stream(x["s"]):
                    x["g"].replay()
            torch.cuda.synchronize()
            for x, w in zip(runs, want):
                assert torch.equal(x["o"], w)
    finally:
        tadm.tadm_model_destroy(m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_a_nan_position_and_of_infinite_scores(dtype):
    """A NaN code reaches the heads that read it and no others; a query whose scores are -inf on whole tiles takes
    the finite keys alone."""
    rng = np.random.default_rng(11)
    H, Hkv, dh, length, n = 4, 2, 64, 300, 5
    pages = random_pages(rng, 6, 1, Hkv, dh)
    pages.side(4, 0, 1, 0)[7] = 0x7f  # K of head 1, position 64 * 2 + 7
    table = np.array([[0, 1, 4, 2, 3]])
    q = torch.from_numpy(rng.normal(size=(1, H, n, dh))).to(DT[dtype])
    k, vt = window(rng, 1, Hkv, 64, dh, dtype)
    k[0, 0, :, 3] = -float("inf")  # head 0: scores of the window are -inf where q[3] > 0 ...
    q[0, :, :, 3] = q[0, :, :, 3].abs() + 0.5
    data, scale, p = to_gpu(pages)
    m = model(dtype, H, Hkv, dh)
    try:
        o, lse = run_attend(m, dtype, p, 0, table, [length], [n], 320, q, k, vt, 64)
    finally:
        tadm.tadm_model_destroy(m)
    o = o.double().cpu().numpy().reshape(n, H, dh)
    assert np.all(np.isnan(o[:, 2:])), "head 1's queries see the NaN key"
    K, V, _ = pages.read(0, table[0], length)
    qb = q[0].double().numpy()
    ref, _ = P.attend(qb[:2], K[:1], V[:1])  # ... so that head 0 has the pages alone
    to, _ = bounds(dtype, qb[:2], K[:1], V[:1])
    assert np.all(np.abs(o[:, :2] - ref) <= to)


def test_attention_offsets_above_32_bits():
    """Pages behind the first 4 GiB of the codes, for every operator."""
    Hkv, dh, layers = 2, 128, 40
    per = layers * Hkv * 2 * 64 * dh
    n_pages = (1 << 32) // per + 3
    rng = np.random.default_rng(3)
    data = torch.zeros(n_pages, layers, Hkv, 2, 64 * dh, dtype=torch.uint8, device="cuda")
    scale = torch.ones(n_pages, layers, Hkv, 2, device="cuda")
    p = tadm.page_set(data, scale)
    m = model("bf16", 4, Hkv, dh)
    try:
        k, vt = window(rng, 1, Hkv, 128, dh, "bf16")
        kd, vd = k.cuda(), vt.cuda()
        t, far = i32([[1, 2]]), i32([[n_pages - 1, n_pages - 2]])
        tadm.tadm_pages_append(m, p, layers - 1, tadm.page_rows(t, 0), kd, vd, 100, 128)
        tadm.tadm_pages_append(m, p, layers - 1, tadm.page_rows(far, 0), kd, vd, 100, 128)
        out = []
        q = torch.from_numpy(rng.normal(size=(1, 4, 3, dh))).to(torch.bfloat16).cuda()
        for tab in (t, far):
            r = tadm.page_rows(tab, 100)
            o = torch.zeros(1, 3, 4 * dh, dtype=torch.bfloat16, device="cuda")
            k2, v2 = torch.zeros_like(kd), torch.zeros_like(vd)
            work = torch.empty(max(tadm.tadm_pages_attend_work(m, r, 3), 16), dtype=torch.uint8, device="cuda")
            tadm.tadm_pages_attend(m, p, layers - 1, r, q, 3, kd, vd, 128, o, None, work)
            tadm.tadm_pages_read(m, p, layers - 1, r, k2, v2, 128)
            out.append((o, k2, v2))
        assert out[0][1].abs().sum() > 0
        for a, b in zip(*out):
            assert torch.equal(a, b)
        tadm.tadm_pages_copy(m, p, [n_pages - 1, n_pages - 2], [3, n_pages - 3])
        assert torch.equal(data[3], data[1]) and torch.equal(data[n_pages - 3], data[2])
    finally:
        tadm.tadm_model_destroy(m)


# ------------------------------------------------------------------ read, copy
@pytest.mark.parametrize("dtype, Hkv, dh, lens", [
    ("f32", 2, 20, [0, 1, 130]), ("f32", 1, 128, [64]), ("bf16", 3, 64, [777, 64, 5, 63]), ("bf16", 2, 128, [300, 191])])
def test_read_is_exact(dtype, Hkv, dh, lens):
    rng = np.random.default_rng(dh)
    B, mp = len(lens), 13
    pages = random_pages(rng, B * mp, 3, Hkv, dh)
    table = rng.permutation(B * mp).reshape(B, mp)
    if max(lens) > 64:
        table[-1, 1] = -1
    data, scale, p = to_gpu(pages)
    cap = 13 * 64
    m = model(dtype, Hkv, Hkv, dh)
    try:
        k = torch.full((B, Hkv, cap, dh), 9.0, dtype=DT[dtype], device="cuda")
        vt = torch.full((B, Hkv, dh, cap), 9.0, dtype=DT[dtype], device="cuda")
        t, ln = i32(table), i32(lens)
        tadm.tadm_pages_read(m, p, 2, tadm.page_rows(t, max(lens), ln), k, vt, cap)
        torch.cuda.synchronize()
    finally:
        tadm.tadm_model_destroy(m)
    k, vt = k.double().cpu().numpy(), vt.double().cpu().numpy()
    for b, length in enumerate(lens):
        K, V, _ = pages.read(2, table[b], length)
        assert np.array_equal(k[b, :, :length], K) and np.array_equal(vt[b, :, :, :length].transpose(0, 2, 1), V)
        assert np.all(k[b, :, length:] == 9.0) and np.all(vt[b, :, :, length:] == 9.0)


@pytest.mark.parametrize("Hkv, dh, layers, n_pages, n", [(1, 4, 1, 5, 2), (2, 20, 3, 40, 17), (4, 128, 2, 1200, 555)])
def test_copy_is_exact(Hkv, dh, layers, n_pages, n):
    rng = np.random.default_rng(n)
    pages = random_pages(rng, n_pages, layers, Hkv, dh)
    ids = rng.permutation(n_pages)
    dst, src = ids[:n], rng.choice(ids[n:], size=n)  # a page may go to several places
    data, scale, p = to_gpu(pages)
    m = model("f32", Hkv, Hkv, dh)
    try:
        tadm.tadm_pages_copy(m, p, src, dst)
        tadm.tadm_pages_copy(m, p, [], [])
        torch.cuda.synchronize()
    finally:
        tadm.tadm_model_destroy(m)
    pages.codes[dst], pages.scales[dst] = pages.codes[src], pages.scales[src]
    assert np.array_equal(data.cpu().numpy(), pages.codes)
    assert np.array_equal(scale.cpu().double().numpy(), pages.scales)


# ------------------------------------------------------------------ streams, capture, refusals
def test_captured_steps_follow_the_lengths():
    """A captured append + attention, replayed while the lengths on the device grow, equals the eager calls."""
    rng = np.random.default_rng(21)
    H, Hkv, dh, B, mp, n = 8, 2, 128, 2, 40, 1
    pages = random_pages(rng, B * mp, 1, Hkv, dh)
    table = i32(rng.permutation(B * mp).reshape(B, mp))
    m = model("bf16", H, Hkv, dh)
    side = torch.cuda.Stream()
    try:
        steps = [(torch.randn(B, H, n, dh, device="cuda").bfloat16(), torch.randn(B, Hkv, 64, dh, device="cuda").bfloat16(),
                  torch.randn(B, Hkv, dh, 64, device="cuda").bfloat16()) for _ in range(5)]
        lens0 = [2047, 62]

        def make():
            data, scale, p = to_gpu(pages)
            s = dict(data=data, scale=scale, p=p, len=i32(lens0), q=steps[0][0].clone(), k=steps[0][1].clone(),
                     vt=steps[0][2].clone(), o=torch.zeros(B, n, H * dh, dtype=torch.bfloat16, device="cuda"),
                     lse=torch.zeros(B, H, n, device="cuda"))
            s["r"] = tadm.page_rows(table, mp * 64, s["len"])
            s["work"] = torch.empty(max(16, tadm.tadm_pages_attend_work(m, s["r"], n)), dtype=torch.uint8, device="cuda")
            return s

        def step(s):
            tadm.tadm_pages_attend(m, s["p"], 0, s["r"], s["q"], n, s["k"], s["vt"], 64, s["o"], s["lse"], s["work"])
            tadm.tadm_pages_append(m, s["p"], 0, s["r"], s["k"], s["vt"], n, 64)
            s["len"].add_(1)

        eager, graph = make(), make()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
            step(graph)
        tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
        for q, k, vt in steps:
            for s in (eager, graph):
                s["q"].copy_(q), s["k"].copy_(k), s["vt"].copy_(vt)
            step(eager)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for name in ("o", "lse", "data", "scale", "len"):
                assert torch.equal(eager[name], graph[name]), name
        # on another stream, behind its own work
        with torch.cuda.stream(side):
            tadm.tadm_set_stream(m, side.cuda_stream)
            eager["q"].copy_(steps[0][0])
            step(eager)
        side.synchronize()
        tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
        graph["q"].copy_(steps[0][0])
        step(graph)
        torch.cuda.synchronize()
        assert torch.equal(eager["o"], graph["o"])
    finally:
        tadm.tadm_model_destroy(m)


def test_refusals_that_need_a_model():
    m = model("bf16", 4, 2, 64)
    try:
        data = torch.zeros(4, 1, 2, 2, 64 * 128, dtype=torch.uint8, device="cuda")
        scale = torch.ones(4, 1, 2, 2, device="cuda")
        t = i32([[0, 1, 2, 3]])
        r = tadm.page_rows(t, 256)
        k = torch.zeros(1, 2, 64, 64, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(tadm.TadmError, match="heads x 128, model of 2 x 64"):
            tadm.tadm_pages_read(m, tadm.page_set(data, scale), 0, tadm.page_rows(t, 64), k, k, 64)
        data = torch.zeros(300, 1, 2, 2, 64 * 64, dtype=torch.uint8, device="cuda")
        scale = torch.ones(300, 1, 2, 2, device="cuda")
        p, t = tadm.page_set(data, scale), i32(np.arange(300)[None])
        r = tadm.page_rows(t, 300 * 64)
        q = torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
        need = tadm.tadm_pages_attend_work(m, r, 1)
        assert need > 0
        for work in (None, torch.empty(need - 1, dtype=torch.uint8, device="cuda")):
            with pytest.raises(tadm.TadmError, match="scratch"):
                tadm.tadm_pages_attend(m, p, 0, r, q, 1, None, None, 0, q.view(1, 1, 256), None, work)
        many = tadm.page_rows(t, 64)
        many.B = 65535
        assert tadm.tadm_pages_attend_work(m, many, 1 << 20) == 0
        with pytest.raises(tadm.TadmError, match="too many"):
            tadm.tadm_pages_attend(m, p, 0, many, q, 1 << 20, None, None, 0, q, None, None)
    finally:
        tadm.tadm_model_destroy(m)
