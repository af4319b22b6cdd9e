"""Many samples of one prompt: forks of a pooled context that attend to what they share together, and a program of its
own that takes pages, attends, appends, draws and gives pages back, as one captured step."""
import numpy as np
import pytest
import torch

import synth
from helpers import dev
from oracle import draw as D
from oracle import pages as P
from test_gpu_pages import bounds, i32, model, random_pages, to_gpu
from test_gpu_pooled import World

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

BIG = {"f32": dict(name="tiny", n_shared=1, n_anchor=1, n_denoise=1, rows=16),
       "bf16": dict(name="block", d_model=256, n_heads=4, n_kv_heads=4, head_dim=128, d_ffn=512, n_anchor=1, n_denoise=1,
                    vocab=1024, rows=16)}


def world(kind, max_seq=4032, pages=260):
    import test_gpu_pooled as T
    spec = dict(BIG[kind])
    rows = spec.pop("rows")
    T.CFGS[kind + " samples"] = spec
    try:
        return World(kind + " samples", B=rows, max_seq=max_seq, pages=pages), rows
    finally:
        del T.CFGS[kind + " samples"]


def prompts(w, n, rows):
    ctx = w.context(B=2)
    for at in range(0, n, 1000):
        w.append(ctx, w.tokens(min(1000, n - at), 30 + at, B=2))
    return ctx, tadm.tadm_context_fork(ctx, [0] * (rows - 7) + [1] * 7)


def close(a, b, tol):
    assert bool(((a - b).abs() <= tol * (1 + b.abs())).all()), float((a - b).abs().max())


@pytest.mark.parametrize("kind, tol", [("f32", 1e-4), ("bf16", 2e-2)])
def test_forks_attend_together(kind, tol):
    """The same logits with and without sharing, before and after the forks part; with groups ruled out the sums have
    another order, so their last bits show that the rows went together."""
    w, rows = world(kind)
    with w:
        src, ctx = prompts(w, 3877, rows)
        z = w.tokens(3, 7, B=rows)
        alone = w.step(ctx, z, B=rows)
        tadm.tadm_context_share(ctx, 1)
        together = w.step(ctx, z, B=rows)
        close(together, alone, tol)
        assert torch.equal(w.step(ctx, z, B=rows), together)
        tadm.tadm_context_share(ctx, 61)  # more pages than they share
        apart = w.step(ctx, z, B=rows)
        close(apart, alone, tol)
        assert not torch.equal(together, apart)
        tadm.tadm_context_share(ctx, 1)
        w.append(ctx, w.tokens(40, 8, B=rows))  # the forks part: the page that the prompt ends in is copied for each
        assert tadm.tadm_context_length(ctx) == 3917 and tadm.tadm_context_length(src) == 3877
        together = w.step(ctx, z, B=rows)
        tadm.tadm_context_share(ctx, 0)
        close(together, w.step(ctx, z, B=rows), tol)
        tadm.tadm_context_truncate(ctx, 100)
        tadm.tadm_context_share(ctx, 1)
        close(w.step(ctx, z, B=rows), (tadm.tadm_context_share(ctx, 0), w.step(ctx, z, B=rows))[1], tol)
        tadm.tadm_context_destroy(ctx)
        tadm.tadm_context_destroy(src)


def test_captured_passes_of_forks():
    """A captured pass that shares, replayed while the pages move and after sharing is off for eager passes."""
    w, rows = world("f32", pages=200)
    with w:
        first = w.context(B=2)
        w.append(first, w.tokens(300, 1, B=2))
        src, ctx = prompts(w, 3840, rows)
        tadm.tadm_context_share(ctx, 1)
        n, z = 2, w.tokens(2, 3, B=rows).to(dev())
        want = w.step(ctx, z.cpu(), B=rows)
        cache = tadm.tadm_cache_create(w.m, rows, n)
        logits = torch.empty(rows, n, w.cfg["vocab"], device=dev())
        nxt = torch.empty(rows, n, dtype=torch.int32, device=dev())

        def run():
            tadm.tadm_anchor_forward(w.m, ctx, z, rows, n, 8, 8, cache)
            tadm.tadm_denoise_step(w.m, ctx, z, rows, n, 0, cache, tadm.step_args(8, 8, 3, 0, 4, 1.0), logits, nxt)

        side, back = torch.cuda.Stream(), torch.cuda.current_stream()
        side.wait_stream(back)
        tadm.tadm_set_stream(w.m, side.cuda_stream)
        with torch.cuda.stream(side):
            run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            with pytest.raises(tadm.TadmError, match="captured"):
                tadm.tadm_context_share(ctx, 2)
            run()
        for i in range(4):
            if i == 1:
                tadm.tadm_context_destroy(first)
                with torch.cuda.stream(side):
                    tadm.tadm_pool_compact(w.pool)
            if i == 3:
                tadm.tadm_context_share(ctx, 0)
            with torch.cuda.stream(side):
                logits.zero_()
                g.replay()
            torch.cuda.synchronize()
            assert torch.equal(logits, want), i
        tadm.tadm_set_stream(w.m, back.cuda_stream)
        tadm.tadm_cache_destroy(cache)
        tadm.tadm_context_destroy(ctx)
        tadm.tadm_context_destroy(src)


def test_share_refusals():
    with World("f32") as w:
        plain, x = tadm.tadm_context_create(w.m, 2, 128), w.context()
        with pytest.raises(tadm.TadmError, match="no pages"):
            tadm.tadm_context_share(plain, 1)
        with pytest.raises(tadm.TadmError, match="min_pages=-1"):
            tadm.tadm_context_share(x, -1)
        tadm.tadm_context_share(x, 3)
        tadm.tadm_context_share(x, 0)
        tadm.tadm_context_destroy(plain)
        tadm.tadm_context_destroy(x)


@pytest.mark.parametrize("rows, says", [(1024, "2.32 threads"), (1025, "B=1025 rows")])
def test_share_refuses_what_no_launch_takes(rows, says):
    """1 024 rows x 4 096 tokens x 32 heads x 32 lanes of the join are 2^32; nothing is allocated or run."""
    cfg = synth.get_config("tiny", dtype="f32", n_heads=32, n_kv_heads=32, head_dim=4, d_model=64, vocab=64)
    m = tadm.tadm_model_create(tadm.make_config(cfg, max_batch=rows, max_seq=4096))
    pool = tadm.tadm_pool_create(m, 1)
    ctx = tadm.tadm_context_create_pooled(m, pool, rows, 64)
    try:
        with pytest.raises(tadm.TadmError, match=says):
            tadm.tadm_context_share(ctx, 1)
        tadm.tadm_context_share(ctx, 0)
    finally:
        tadm.tadm_context_destroy(ctx)
        tadm.tadm_pool_destroy(pool)
        tadm.tadm_model_destroy(m)


@pytest.mark.parametrize("dtype, H, Hkv, dh", [("f32", 4, 4, 16), ("bf16", 16, 16, 128)])
def test_a_captured_step_of_samples(dtype, H, Hkv, dh):
    """Each replay takes pages for one to three tokens a row, attends over the prompt's shared pages, the row's own and the new
    tokens, appends these, draws a token a row, and advances the lengths; at last the newest tokens are given back."""
    rng = np.random.default_rng(23)
    B, whole, n, V, mp, free = 16, 40, 3, 64, 46, 30
    size = whole + B + free
    pages = random_pages(rng, size, 1, Hkv, dh)
    ids = rng.permutation(size).tolist()
    prompt = [ids.pop() for _ in range(whole)]
    table = [prompt + [ids.pop()] + [-1] * (mp - whole - 1) for _ in range(B)]  # each with a page of its own behind
    lens = [64 * whole + int(x) for x in rng.integers(40, 65, size=B)]
    data, scale, p = to_gpu(pages)
    m = model(dtype, H, Hkv, dh)  # vocabulary 64
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    t, ln, nn, granted = i32(table), i32(lens), i32([0] * B), i32([0] * B)
    stack_ids, state = i32(ids + [-1] * (size - free)), i32([free, 0, 0, 0])
    stack, slots = tadm.page_stack(stack_ids, state), torch.zeros(B, n, dtype=torch.int64, device="cuda")
    take, rows = tadm.page_rows(t, mp * 64, ln, nn), tadm.page_rows(t, mp * 64, ln, granted)
    plan_data = torch.empty(tadm.tadm_pages_plan_bytes(m, rows, n), dtype=torch.uint8, device="cuda")
    plan = tadm.page_plan(plan_data)
    work = torch.empty(tadm.tadm_pages_attend_shared_work(m, rows, n), dtype=torch.uint8, device="cuda")
    q = torch.zeros(B, H, n, dh, dtype=dt, device="cuda")
    k, vt = torch.zeros(B, Hkv, 64, dh, dtype=dt, device="cuda"), torch.zeros(B, Hkv, dh, 64, dtype=dt, device="cuda")
    o = torch.zeros(B, n, H * dh, dtype=dt, device="cuda")
    logits, u = torch.zeros(B, V, device="cuda"), torch.zeros(B, device="cuda")
    token, logp = i32([0] * B), torch.zeros(B, device="cuda")
    settings = dict(temperature=rng.choice([0.0, 0.7, 1.0], size=B).astype(np.float32), top_k=rng.choice([0, 5, 20], size=B),
                    top_p=rng.choice([1.0, 0.8], size=B).astype(np.float32))
    on_dev = {a: torch.from_numpy(v.astype(np.int32 if a == "top_k" else np.float32)).cuda() for a, v in settings.items()}
    drawn = tadm.row_settings(**on_dev)
    draw_work = torch.empty(max(16, tadm.tadm_sample_rows_work(m, B)), dtype=torch.uint8, device="cuda")
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    side.wait_stream(main)
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.stream(side):
            tadm.tadm_set_stream(m, side.cuda_stream)
            with torch.cuda.graph(graph, stream=side):
                tadm.tadm_pages_assign(m, stack, take, n, granted, slots)
                tadm.tadm_pages_share(m, rows, n, 1, plan)
                tadm.tadm_pages_attend_shared(m, p, 0, rows, plan, q, n, k, vt, 64, o, None, work)
                tadm.tadm_pages_append(m, p, 0, rows, k, vt, n, 64)
                tadm.tadm_sample_rows(m, logits, drawn, u, token, logp, draw_work)
                ln.add_(granted)
            tadm.tadm_set_stream(m, main.cuda_stream)
        main.wait_stream(side)
        left, ref_ids = free, list(ids)
        for step in range(12):
            news = rng.integers(0 if step % 3 else 1, n + 1, size=B).tolist()
            qs = torch.from_numpy(rng.normal(size=tuple(q.shape))).to(dt)
            ks, vs = torch.from_numpy(rng.normal(size=tuple(k.shape))).to(dt), torch.from_numpy(rng.normal(size=tuple(vt.shape))).to(dt)
            ls, us = (rng.normal(size=(B, V)) * 2).astype(np.float32), rng.random(B).astype(np.float32)
            for d, h in ((nn, i32(news)), (q, qs), (k, ks), (vt, vs), (logits, torch.from_numpy(ls)), (u, torch.from_numpy(us))):
                d.copy_(h)
            got_all, ref_slots, left = P.assign(table, lens, news, ref_ids, left, size)
            graph.replay()
            torch.cuda.synchronize()
            assert granted.tolist() == got_all and state.tolist() == [left, 0, 0, 0] and t.tolist() == table
            assert slots.tolist() == [s + [-1] * (n - len(s)) for s in ref_slots]
            got = o.double().cpu().numpy().reshape(B, n, H, dh)
            for b, g in enumerate(got_all):
                if g == 0:
                    continue
                pk, pv, _ = pages.read(0, table[b], lens[b])
                kb, vb = ks[b, :, :g].double().numpy(), vs[b, :, :, :g].double().numpy().transpose(0, 2, 1)
                pk, pv, qb = np.concatenate([pk, kb], 1), np.concatenate([pv, vb], 1), qs[b, :, :g].double().numpy()
                assert (np.abs(got[b, :g] - P.attend(qb, pk, pv)[0]) <= bounds(dtype, qb, pk, pv)[0]).all(), (step, b)
                pages.append(0, table[b], lens[b], kb, vb)
            lens = [a + g for a, g in zip(lens, got_all)]
            assert ln.tolist() == lens
            assert np.array_equal(data.cpu().numpy(), pages.codes) and np.array_equal(scale.cpu().double().numpy(), pages.scales)
            assert token.tolist() == [D.draw(ls[b], us[b], **{a: v[b] for a, v in settings.items()})[0] for b in range(B)]
        lens = [a - g for a, g in zip(lens, got_all)]
        ln.copy_(i32(lens))
        tadm.tadm_pages_release(m, stack, rows, n)
        left = P.release(table, lens, got_all, ref_ids, left, size)
        torch.cuda.synchronize()
        assert state.tolist() == [left, 0, 0, 0] and t.tolist() == table and stack_ids[:left].tolist() == ref_ids[:left]
    finally:
        tadm.tadm_set_stream(m, main.cuda_stream)
        tadm.tadm_model_destroy(m)
