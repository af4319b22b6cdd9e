"""What a page pool and its contexts must not do to one another, and the calls that they refuse."""
import numpy as np
import pytest
import torch

from oracle import pages as P

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_pages import bounds, i32, window  # noqa: E402
from test_gpu_pooled import World, same  # noqa: E402
from test_gpu_pooled import test_passes_on_a_pooled_context as passes  # noqa: E402
from helpers import dev  # noqa: E402


def pages_seen(w, ctx, layer=0):
    """Which places of each row's table name a page, as an operator over all of them finds them ([B, max_pages])."""
    r, hk, dh = tadm.tadm_context_rows(ctx), w.cfg["n_kv_heads"], w.cfg["head_dim"]
    r.len = r.max_pages * 64
    k = torch.full((r.B, hk, r.len, dh), 7.0, dtype=w.dt, device=dev())
    vt = torch.full((r.B, hk, dh, r.len), 7.0, dtype=w.dt, device=dev())
    tadm.tadm_pages_read(w.m, tadm.tadm_pool_pages(w.pool), layer, r, k, vt, r.len)
    return (k.abs().amax((1, 3)) > 0).view(r.B, -1, 64).any(2).tolist()  # an absent page reads as zeros


def test_calls_after_an_allocation_that_failed():
    """A pool or a context that does not fit the device is refused, and the next calls, which are sound, succeed."""
    with World("bf16 128") as w:
        ctx, plain = w.context(), tadm.tadm_context_create(w.m, 2, 128)
        w.append(ctx, w.tokens(70, 1))
        before = w.read(ctx)
        for call in (lambda: tadm.tadm_pool_create(w.m, 4_000_000), lambda: tadm.tadm_pool_resize(w.pool, 4_000_000)):
            for after in (lambda: w.append(plain, w.tokens(5, 2)), lambda: w.append(ctx, w.tokens(5, 2)), lambda: w.read(ctx)):
                with pytest.raises(tadm.TadmError) as e:
                    call()
                assert e.value.status == tadm.TADM_ERR_OOM
                after()
        assert tadm.tadm_pool_size(w.pool) == 40 and tadm.tadm_context_length(ctx) == 80
        tadm.tadm_context_truncate(ctx, 64)
        assert all((x[:, :, :64] == y).all() for u, v in zip(before, w.read(ctx)) for x, y in zip(u, v))
        tadm.tadm_context_destroy(ctx)
        tadm.tadm_context_destroy(plain)


@pytest.mark.parametrize("kind", ["f32", "bf16 128"])
def test_a_table_names_the_pages_of_its_context_alone(kind):
    """On the device too, places that never had a page or whose page was given back name none, whoever has it now."""
    with World(kind, pages=24) as w:
        filled = w.context()
        w.append(filled, w.tokens(300, 1))  # 10 pages, none of them empty when it lets go of them
        tadm.tadm_context_destroy(filled)
        ctx, other = w.context(), w.context(B=1)
        holds = lambda n: [[i < n for i in range(7)]] * 2  # noqa: E731
        assert pages_seen(w, ctx) == holds(0)
        w.append(ctx, w.tokens(330, 2))
        assert pages_seen(w, ctx) == holds(6)
        kid = tadm.tadm_context_fork(ctx, [1, 0])
        assert pages_seen(w, kid) == holds(6)
        for keep, n in ((330, 6), (321, 6), (320, 5), (193, 4), (128, 2), (100, 2)):
            tadm.tadm_context_truncate(ctx, keep)
            assert pages_seen(w, ctx) == holds(n), keep
        tadm.tadm_context_destroy(kid)
        w.append(other, w.tokens(400, 3, 1))  # takes pages that ctx had
        assert pages_seen(w, ctx) == holds(2)
        w.append(ctx, w.tokens(100, 4))
        assert pages_seen(w, ctx) == holds(4)
        tadm.tadm_context_reset(ctx)
        assert pages_seen(w, ctx) == holds(0)
        for x in (ctx, other):
            tadm.tadm_context_destroy(x)
        assert tadm.tadm_pool_free_pages(w.pool) == 24


@pytest.mark.parametrize("kind", ["f32", "bf16 128"])
def test_a_captured_call_after_a_rollback(kind):
    """Attention over a context's rows, captured at 130 positions and replayed after the context fell back to 64
    and another took the pages it gave back: equals the oracle over the 64 positions, replay after replay; what
    gives back or takes pages is refused under capture and changes nothing."""
    with World(kind) as w:
        ctx, other = w.context(), w.context()
        w.append(ctx, w.tokens(130, 1))
        H, hk, dh, n = w.cfg["n_heads"], w.cfg["n_kv_heads"], w.cfg["head_dim"], 5
        q = torch.randn(w.B, H, n, dh, device=dev()).to(w.dt)
        o = torch.zeros(w.B, n, H * dh, dtype=w.dt, device=dev())
        p, r = tadm.tadm_pool_pages(w.pool), tadm.tadm_context_rows(ctx)
        work = torch.empty(max(16, tadm.tadm_pages_attend_work(w.m, r, n)), dtype=torch.uint8, device=dev())
        call = lambda: tadm.tadm_pages_attend(w.m, p, 1, r, q, n, None, None, 0, o, None, work)  # noqa: E731

        def check(length):
            k, v = w.read(ctx)[1]
            for b in range(w.B):
                qb = q[b].double().cpu().numpy()
                ref, _ = P.attend(qb, k[b][:, :length], v[b][:, :length])
                to, _ = bounds("f32" if w.dt == torch.float32 else "bf16", qb, k[b][:, :length], v[b][:, :length])
                assert np.all(np.abs(o[b].double().cpu().numpy().reshape(n, H, dh) - ref) <= to)

        call()
        check(130)
        side, back = torch.cuda.Stream(), torch.cuda.current_stream()
        free = tadm.tadm_pool_free_pages(w.pool)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            tadm.tadm_set_stream(w.m, side.cuda_stream)
            for refused in (lambda: tadm.tadm_context_truncate(ctx, 128), lambda: tadm.tadm_context_reset(ctx),
                            lambda: w.context()):
                with pytest.raises(tadm.TadmError, match="captured") as e:
                    refused()
                assert e.value.status == tadm.TADM_ERR_STATE
            tadm.tadm_context_truncate(ctx, 130)  # gives nothing back
            tadm.tadm_context_reset(other)
            call()
        tadm.tadm_set_stream(w.m, back.cuda_stream)
        assert tadm.tadm_context_length(ctx) == 130 and tadm.tadm_pool_free_pages(w.pool) == free
        for length in (130, 128, 64, 64):
            tadm.tadm_context_truncate(ctx, length)
            tadm.tadm_context_reset(other)
            w.append(other, w.tokens(250, length))
            o.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            check(length)
        for x in (ctx, other):
            tadm.tadm_context_destroy(x)


def test_forks_under_capture_are_refused():
    """A fork within a capture is refused, leaves no trace in the pool and does not disturb the capture; forked
    before it, the new context runs the captured pass like the old one, while the old one goes on."""
    with World("bf16 128") as w:
        root = w.context()
        w.append(root, w.tokens(100, 1))
        kid = tadm.tadm_context_fork(root, [0, 1])
        B, n, z = w.B, 16, w.tokens(16, 2).to(dev())
        want, free = w.step(root, z), tadm.tadm_pool_free_pages(w.pool)
        cache = tadm.tadm_cache_create(w.m, B, n)
        logits = torch.empty(B, n, w.cfg["vocab"], device=dev())
        nxt = torch.empty(B, n, dtype=torch.int32, device=dev())
        side, back = torch.cuda.Stream(), torch.cuda.current_stream()
        tadm.tadm_set_stream(w.m, side.cuda_stream)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for rows in ([0, 1], [1]):
                with pytest.raises(tadm.TadmError, match="captured") as e:
                    tadm.tadm_context_fork(root, rows)
                assert e.value.status == tadm.TADM_ERR_STATE
            tadm.tadm_anchor_forward(w.m, kid, z, B, n, 8, 8, cache)
            tadm.tadm_denoise_step(w.m, kid, z, B, n, 0, cache, tadm.step_args(8, 8, 3, 0, 4, 1.0), logits, nxt)
        tadm.tadm_set_stream(w.m, back.cuda_stream)
        assert tadm.tadm_pool_free_pages(w.pool) == free
        for i in range(4):
            w.append(root, w.tokens(10, 20 + i))  # copies the page that it shares with the fork, then goes on alone
            logits.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(logits, want), i
        tadm.tadm_cache_destroy(cache)
        for x in (root, kid):
            tadm.tadm_context_destroy(x)
        assert tadm.tadm_pool_free_pages(w.pool) == 40


@pytest.mark.parametrize("kind", ["f32", "bf16 128"])
def test_operators_on_the_rows_of_a_context(kind):
    """Reading and attending work on a pool's pages with a context's rows; appending is refused, also to a part of
    the table, and neither the context nor a fork that shares its pages changes.  Rows and pages of the program's own
    are appended to as ever."""
    with World(kind) as w:
        first, ctx = w.context(), w.context()
        w.append(first, w.tokens(70, 1))
        w.append(ctx, w.tokens(150, 2))
        kid = tadm.tadm_context_fork(ctx, [0, 1])
        before = w.read(ctx)
        p, r = tadm.tadm_pool_pages(w.pool), tadm.tadm_context_rows(ctx)
        H, hk, dh, n = w.cfg["n_heads"], w.cfg["n_kv_heads"], w.cfg["head_dim"], 6
        name = "f32" if w.dt == torch.float32 else "bf16"
        k, vt = window(np.random.default_rng(3), w.B, hk, 64, dh, name, 9.0)
        q, kd, vd = torch.randn(w.B, H, n, dh, device=dev()).to(w.dt), k.to(dev()), vt.to(dev())
        work = torch.empty(max(16, tadm.tadm_pages_attend_work(w.m, r, n)), dtype=torch.uint8, device=dev())
        for layer in range(w.layers):
            k2, v2 = torch.zeros(w.B, hk, 192, dh, dtype=w.dt, device=dev()), torch.zeros(w.B, hk, dh, 192, dtype=w.dt, device=dev())
            tadm.tadm_pages_read(w.m, p, layer, r, k2, v2, 192)
            K, V = before[layer]
            assert np.array_equal(k2[:, :, :150].double().cpu().numpy(), K)
            assert np.array_equal(v2[..., :150].transpose(2, 3).double().cpu().numpy(), V)
            o = torch.zeros(w.B, n, H * dh, dtype=w.dt, device=dev())
            tadm.tadm_pages_attend(w.m, p, layer, r, q, n, kd, vd, 64, o, None, work)
            for b in range(w.B):
                qb = q[b].double().cpu().numpy()
                Kb = np.concatenate([K[b], k[b, :, :n].double().numpy()], 1)
                Vb = np.concatenate([V[b], vt[b, :, :, :n].double().numpy().transpose(0, 2, 1)], 1)
                ref, _ = P.attend(qb, Kb, Vb)
                to, _ = bounds(name, qb, Kb, Vb)
                assert np.all(np.abs(o[b].double().cpu().numpy().reshape(n, H, dh) - ref) <= to)
        for skip, length in ((0, 150), (0, 40), (0, 192), (7, 0), (13, 0)):
            part = tadm.tadm_context_rows(ctx)
            part.table_dev, part.len = part.table_dev + 4 * skip, length
            part.B, part.max_pages = (2, 7) if skip == 0 else (1, 14 - skip)
            with pytest.raises(tadm.TadmError, match="tadm_context_append") as e:
                tadm.tadm_pages_append(w.m, p, 0, part, kd, vd, 8, 64)
            assert e.value.status == tadm.TADM_ERR_STATE
        data = torch.zeros(2, 1, hk, 2, 64 * dh, dtype=torch.uint8, device=dev())
        scale, table = torch.ones(2, 1, hk, 2, device=dev()), i32([[0], [1]])
        tadm.tadm_pages_append(w.m, tadm.page_set(data, scale), 0, tadm.page_rows(table, 0), kd, vd, 64, 64)
        assert (data != 0).any() and (scale != 1).all()
        for x in (ctx, kid):
            assert same(before, w.read(x))
        for x in (first, ctx, kid):
            tadm.tadm_context_destroy(x)


@pytest.mark.parametrize("kind", ["f32", "bf16 64"])
def test_a_rollback_to_whole_pages_leaves_no_trace(kind):
    """Positions appended and dropped again at a page's end, then others: reads and runs bit for bit as a context that
    never had them."""
    with World(kind) as w:
        a, direct = w.context(), w.context()
        first, last, z = w.tokens(64, 1), w.tokens(36, 2), w.tokens(12, 3)
        for x in (a, direct):
            w.append(x, first)
        w.append(a, w.tokens(30, 4))
        w.append(a, w.tokens(90, 5))
        tadm.tadm_context_truncate(a, 64)
        for x in (a, direct):
            w.append(x, last)
        assert same(w.read(a), w.read(direct))
        assert torch.equal(w.step(a, z), w.step(direct, z))
        for x in (a, direct):
            tadm.tadm_context_destroy(x)


@pytest.mark.parametrize("kind", ["f32", "bf16 64", "bf16 128"])
@pytest.mark.parametrize("keep, shared", [(70, False), (70, True), (127, True), (65, False)])
def test_a_rollback_inside_a_page(kind, keep, shared):
    """130 positions, cut inside the second page, then 20 others: layer 0, whose K, V depend on tokens and positions
    alone, holds what the page oracle makes of a plain context's K, V (the kept page's scale and rounding
    included).  A fork on the same pages reads as before, and, cut and continued like the other, reads alike."""
    with World(kind) as w:
        x, plain = w.context(), tadm.tadm_context_create(w.m, w.B, 448)
        hk, dh = w.cfg["n_kv_heads"], w.cfg["head_dim"]
        pages = [P.Pages(np.zeros((3, 1, hk, 2, 64 * dh), np.uint8), np.ones((3, 1, hk, 2))) for _ in range(w.B)]

        def append(at, tok):
            for c in (x, plain):
                w.append(c, tok)
            k, v = w.read(plain)[0]
            for b in range(w.B):
                pages[b].append(0, [0, 1, 2], at, k[b][:, at:], v[b][:, at:])

        append(0, w.tokens(130, 1))
        whole, kid = w.read(x), tadm.tadm_context_fork(x, [0, 1]) if shared else None
        for c in (x, plain):
            tadm.tadm_context_truncate(c, keep)
        append(keep, w.tokens(20, 2))
        got = w.read(x)
        for b in range(w.B):
            K, V, _ = pages[b].read(0, [0, 1, 2], keep + 20)
            assert np.array_equal(got[0][0][b], K) and np.array_equal(got[0][1][b], V), b
        if shared:
            assert same(whole, w.read(kid))
            tadm.tadm_context_truncate(kid, keep)
            w.append(kid, w.tokens(20, 2))
            assert same(got, w.read(kid)) and same(got, w.read(x))
            tadm.tadm_context_destroy(kid)
        for c in (x, plain):
            tadm.tadm_context_destroy(c)
        assert tadm.tadm_pool_free_pages(w.pool) == 40


@pytest.mark.parametrize("kind", ["f32", "bf16 64", "bf16 128"])
@pytest.mark.parametrize("pieces", [(300, 100), (413,)])
def test_passes_behind_a_prompt(kind, pieces):
    """Prompts of several tiles appended at once, and once more behind them, then a refresh and a step, against the
    oracle."""
    passes(kind, pieces)
