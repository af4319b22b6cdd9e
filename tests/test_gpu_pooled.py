"""Contexts whose K, V are pages of a pool: the passes of the model on them, sharing, rollback,
compaction and exhaustion.

The reference of a pass is the oracle on the values that the pages hold (read back through
tadm_context_read); what is appended is checked against the oracle's own K, V to the rounding
of the format.  Contexts reached on different ways (forked, rolled back, moved) are compared
bit for bit with contexts built directly."""
import numpy as np
import pytest
import torch

import synth
from helpers import dev, gpu_model, oracle_net, rows_close

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

CFGS = {
    "f32": dict(name="tiny", n_kv_heads=2, n_shared=1, n_anchor=1, n_denoise=1),
    "f32 paired": dict(name="tiny", head_dim=20, n_heads=2, n_kv_heads=2, d_model=64, fusion_kind="paired", fusion_rank=32,
                       paired_heads=4),
    "bf16 64": dict(name="block", d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ffn=1024, n_anchor=1, n_denoise=1,
                    vocab=4096),
    "bf16 128": dict(name="block", d_model=256, n_heads=4, n_kv_heads=4, head_dim=128, d_ffn=512, n_anchor=1, n_denoise=2,
                     vocab=1024),
}


class World:
    """A model with its weights on the GPU and in the oracle, and a pool."""

    def __init__(self, kind, B=2, max_seq=448, pages=40):
        spec = dict(CFGS[kind])
        self.cfg = synth.get_config(spec.pop("name"), **spec)
        self.B, self.dt = B, torch.float32 if self.cfg["dtype"] == "f32" else torch.bfloat16
        tensors = synth.make_weights(self.cfg, perturb=True)
        self.net = oracle_net(self.cfg, tensors)
        self.m = gpu_model(self.cfg, tensors, B, max_seq)
        self.max_seq, self.layers = max_seq, synth.configs.n_layers(self.cfg)
        self.pool = tadm.tadm_pool_create(self.m, pages)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        torch.cuda.synchronize()
        if exc[0] is None:
            tadm.tadm_pool_destroy(self.pool)
        tadm.tadm_model_destroy(self.m)

    def context(self, B=None, cap=None):
        return tadm.tadm_context_create_pooled(self.m, self.pool, B or self.B, cap or self.max_seq)

    def tokens(self, n, seed, B=None):
        g = torch.Generator().manual_seed(seed)
        return torch.randint(0, self.cfg["vocab"], (B or self.B, n), generator=g, dtype=torch.int32)

    def append(self, ctx, tok):
        tadm.tadm_context_append(self.m, ctx, tok.to(dev()), tok.shape[0], tok.shape[1])

    def read(self, ctx, B=None):
        """Per layer (K [B, Hkv, len, dh], V the same) of a context."""
        B = B or self.B
        cap, n = tadm.tadm_context_capacity(ctx), tadm.tadm_context_length(ctx)
        out = []
        for li in range(self.layers):
            k = torch.zeros(B, self.cfg["n_kv_heads"], cap, self.cfg["head_dim"], dtype=self.dt, device=dev())
            vt = torch.zeros(B, self.cfg["n_kv_heads"], self.cfg["head_dim"], cap, dtype=self.dt, device=dev())
            tadm.tadm_context_read(ctx, li, k, vt)
            out.append((k[:, :, :n].double().cpu().numpy(), vt[..., :n].transpose(2, 3).double().cpu().numpy()))
        return out

    def step(self, ctx, z, B=None):
        """Logits of a refresh and a step on the window z [B, n]."""
        B, n = B or self.B, z.shape[1]
        cache = tadm.tadm_cache_create(self.m, B, n)
        logits = torch.empty(B, n, self.cfg["vocab"], device=dev())
        nxt = torch.empty(B, n, dtype=torch.int32, device=dev())
        zd = z.to(dev())
        tadm.tadm_anchor_forward(self.m, ctx, zd, B, n, 8, 8, cache)
        tadm.tadm_denoise_step(self.m, ctx, zd, B, n, 0, cache, tadm.step_args(8, 8, 3, 0, 4, 1.0), logits, nxt)
        torch.cuda.synchronize()
        tadm.tadm_cache_destroy(cache)
        return logits


def same(a, b):
    return all(np.array_equal(x, y) for u, v in zip(a, b) for x, y in zip(u, v))


@pytest.mark.parametrize("kind", list(CFGS))
@pytest.mark.parametrize("pieces", [(70,), (64, 1, 40), (1, 1, 126)])
def test_passes_on_a_pooled_context(kind, pieces):
    """Append in pieces that end inside and at the end of pages, then a refresh and a step on a window."""
    tol = 1e-4 if kind.startswith("f32") else 2e-2
    with World(kind) as w:
        ctx = w.context()
        tok = w.tokens(sum(pieces), 5)
        at = 0
        for n in pieces:
            before = w.read(ctx)
            pos = np.arange(at, at + n)
            w.append(ctx, tok[:, at:at + n])
            after = w.read(ctx)
            for b in range(w.B):
                kv = {li: (k[b].transpose(1, 0, 2), v[b].transpose(1, 0, 2)) for li, (k, v) in enumerate(before)} if at else None
                fresh = w.net.fresh_kv(tok[b, at:at + n].numpy(), pos, kv)
                for li in range(w.layers):
                    for side in range(2):
                        ref = fresh[li][side].transpose(1, 0, 2)
                        got = after[li][side][b][:, at:]
                        # a rounding of the format (half a step: 2^-4 of a normal value, 2^-10 of the scale of a
                        # subnormal one; a page's scale is at most 2 max / 448 = max 2^-7) and the pass's own error
                        top = np.abs(after[li][side][b]).max()
                        assert np.all(np.abs(got - ref) <= 2.0 ** -4 * np.abs(ref) + top * 2.0 ** -17 + tol * (1 + np.abs(ref)) * 1.1)
            at += n
        assert tadm.tadm_context_length(ctx) == at
        z = w.tokens(33, 6)
        z[torch.rand(z.shape, generator=torch.Generator().manual_seed(1)) < 0.6] = w.cfg["vocab"]
        logits, kv, pos = w.step(ctx, z), w.read(ctx), np.arange(at, at + 33)
        for b in range(w.B):
            c_kv = {li: (k[b].transpose(1, 0, 2), v[b].transpose(1, 0, 2)) for li, (k, v) in enumerate(kv)}
            c = w.net.shared(z[b].numpy(), pos, c_kv)
            cache = w.net.anchor_cache(c, pos, c_kv)
            xf = w.net.denoise(w.net.fuse(c, cache), pos, c_kv)
            rows_close(logits[b].cpu().numpy(), w.net.head(xf), what=f"{kind} logits row {b}", rtol=tol, atol=tol)
        tadm.tadm_context_destroy(ctx)
        assert tadm.tadm_pool_free_pages(w.pool) == 40


@pytest.mark.parametrize("kind", ["f32", "bf16 128"])
@pytest.mark.parametrize("P", [64, 70])
def test_forks_share_pages_and_part_when_they_append(kind, P):
    """Candidates forked from one prompt, each continued on its own, equal contexts that were built from the start;
    the prompt's context stays as it was; full pages are shared."""
    with World(kind) as w:
        root = w.context()
        prompt = w.tokens(P, 1)
        w.append(root, prompt)
        base = w.read(root)
        used = 40 - tadm.tadm_pool_free_pages(w.pool)
        assert used == 2 * -(-P // 64)
        kids, conts = [], []
        for i in range(3):
            kid = tadm.tadm_context_fork(root, [1, 1] if i == 2 else [0, 1])
            assert tadm.tadm_context_length(kid) == P and tadm.tadm_context_capacity(kid) == tadm.tadm_context_capacity(root)
            kids.append(kid)
            conts.append(w.tokens(5 + 30 * i, 10 + i))
        assert 40 - tadm.tadm_pool_free_pages(w.pool) == used  # a fork takes no page
        for kid, tok in zip(kids, conts):
            w.append(kid, tok)
        assert same(w.read(root), base)
        for i, (kid, tok) in enumerate(zip(kids, conts)):
            own = w.context()
            w.append(own, prompt if i < 2 else prompt[[1, 1]])
            w.append(own, tok)
            assert same(w.read(own), w.read(kid)), f"fork {i}"
            z = w.tokens(9, 3)
            assert torch.equal(w.step(own, z), w.step(kid, z))
            tadm.tadm_context_destroy(own)
        # the prompt goes first; the last holder of a page keeps it without a copy
        tadm.tadm_context_destroy(root)
        w.append(kids[0], w.tokens(3, 50))
        for kid in kids:
            tadm.tadm_context_destroy(kid)
        assert tadm.tadm_pool_free_pages(w.pool) == 40


@pytest.mark.parametrize("kind", ["f32", "bf16 64"])
def test_rollback_compaction_and_resize(kind):
    """truncate, then other tokens: equal to never having appended the dropped ones where the pages' scales did not
    grow by them; contexts read and run the same bit for bit after the pool was packed and resized."""
    with World(kind) as w:
        a, b, c = w.context(), w.context(B=1), w.context()
        for x, seed, n, rows in ((a, 1, 100, 2), (b, 2, 200, 1), (c, 3, 130, 2)):
            w.append(x, w.tokens(n, seed, rows))
        kept = w.read(a)
        w.append(a, w.tokens(90, 4))
        tadm.tadm_context_truncate(a, 128)
        tadm.tadm_context_truncate(a, 128)
        assert tadm.tadm_context_length(a) == 128
        with pytest.raises(tadm.TadmError):
            tadm.tadm_context_truncate(a, 129)
        tadm.tadm_context_truncate(a, 64)  # whole pages: nothing that was dropped has left a trace
        for (k0, v0), (k1, v1) in zip(kept, w.read(a)):
            assert np.array_equal(k0[:, :, :64], k1) and np.array_equal(v0[:, :, :64], v1)
        w.append(a, w.tokens(36, 9))
        fork = tadm.tadm_context_fork(c, [1])
        before = [w.read(a), w.read(c), w.read(fork, B=1)]
        z = w.tokens(12, 8)
        logits = [w.step(a, z), w.step(c, z)]
        tadm.tadm_context_destroy(b)  # leaves holes
        free = tadm.tadm_pool_free_pages(w.pool)
        tadm.tadm_pool_compact(w.pool)
        tadm.tadm_pool_compact(w.pool)
        held = 40 - tadm.tadm_pool_free_pages(w.pool)
        assert held == 40 - free
        for size in (held, 64, held + 3):
            assert same(before[0], w.read(a)) and same(before[1], w.read(c)) and same(before[2], w.read(fork, B=1))
            assert torch.equal(logits[0], w.step(a, z)) and torch.equal(logits[1], w.step(c, z))
            tadm.tadm_pool_resize(w.pool, size)
            assert tadm.tadm_pool_size(w.pool) == size and tadm.tadm_pool_free_pages(w.pool) == size - held
        with pytest.raises(tadm.TadmError):
            tadm.tadm_pool_resize(w.pool, held - 1)
        rows = tadm.tadm_context_rows(c)
        assert (rows.B, rows.len, rows.max_pages) == (2, 130, 448 // 64)
        w.append(c, w.tokens(20, 12))
        assert same(before[2], w.read(fork, B=1))
        for x in (a, c, fork):
            tadm.tadm_context_reset(x)
        assert tadm.tadm_pool_free_pages(w.pool) == held + 3
        with pytest.raises(tadm.TadmError, match="still use"):
            tadm.tadm_pool_destroy(w.pool)
        for x in (a, c, fork):
            tadm.tadm_context_destroy(x)


def test_a_pool_that_runs_out():
    """An append that needs more pages than are free changes nothing and can be made when there are."""
    with World("f32", pages=5) as w:
        a, b = w.context(), w.context(B=1)
        w.append(a, w.tokens(70, 1))  # 4 pages
        w.append(b, w.tokens(64, 2, 1))
        fork = tadm.tadm_context_fork(a, [0, 0])
        held = [w.read(a), w.read(b, 1), w.read(fork)]
        for x, n, rows in ((a, 60, 2), (b, 1, 1), (fork, 1, 2)):
            with pytest.raises(tadm.TadmError) as e:
                w.append(x, w.tokens(n, 7, rows))
            assert e.value.status == tadm.TADM_ERR_OOM
        assert same(held[0], w.read(a)) and same(held[1], w.read(b, 1)) and same(held[2], w.read(fork))
        assert tadm.tadm_pool_free_pages(w.pool) == 0 and tadm.tadm_context_length(fork) == 70
        tadm.tadm_context_destroy(b)
        with pytest.raises(tadm.TadmError):
            w.append(fork, w.tokens(1, 7))  # two copies, one page
        tadm.tadm_pool_resize(w.pool, 6)
        w.append(fork, w.tokens(1, 7))
        assert tadm.tadm_pool_free_pages(w.pool) == 0 and same(held[0], w.read(a))
        for x in (a, fork):
            tadm.tadm_context_destroy(x)


def test_pooled_refusals():
    with World("f32") as w, World("f32") as other:
        plain = tadm.tadm_context_create(w.m, 2, 128)
        x = w.context()
        with pytest.raises(tadm.TadmError, match="another model"):
            tadm.tadm_context_create_pooled(other.m, w.pool, 1, 64)
        for B, cap in ((0, 64), (3, 64), (1, 0), (1, 449)):
            with pytest.raises(tadm.TadmError):
                tadm.tadm_context_create_pooled(w.m, w.pool, B, cap)
        with pytest.raises(tadm.TadmError, match="pooled"):
            tadm.tadm_context_fork(plain, [0])
        with pytest.raises(tadm.TadmError, match="no pages"):
            tadm.tadm_context_rows(plain)
        for rows in ([], [2], [-1], [0, 1, 1]):
            with pytest.raises(tadm.TadmError):
                tadm.tadm_context_fork(x, rows)
        w.append(plain, w.tokens(100, 1))
        tadm.tadm_context_truncate(plain, 40)
        assert tadm.tadm_context_length(plain) == 40
        for n in (0, -1):
            with pytest.raises(tadm.TadmError):
                tadm.tadm_pool_create(w.m, n)
        tadm.tadm_context_destroy(plain)
        tadm.tadm_context_destroy(x)


def test_captured_passes_follow_the_pages():
    """A captured pass over a pooled context, replayed while its pages move, equals the eager one; appending
    and moving pages are refused under capture and leave the context as it was."""
    with World("bf16 128") as w:
        first, ctx = w.context(), w.context()
        w.append(first, w.tokens(130, 1))
        w.append(ctx, w.tokens(100, 2))
        B, n, z = w.B, 24, w.tokens(24, 3).to(dev())
        want = w.step(ctx, z)
        cache = tadm.tadm_cache_create(w.m, B, n)
        logits = torch.empty(B, n, w.cfg["vocab"], device=dev())
        nxt = torch.empty(B, n, dtype=torch.int32, device=dev())
        more = w.tokens(70, 4).to(dev())

        def run():
            tadm.tadm_anchor_forward(w.m, ctx, z, B, n, 8, 8, cache)
            tadm.tadm_denoise_step(w.m, ctx, z, B, n, 0, cache, tadm.step_args(8, 8, 3, 0, 4, 1.0), logits, nxt)

        side, back = torch.cuda.Stream(), torch.cuda.current_stream()
        side.wait_stream(back)
        tadm.tadm_set_stream(w.m, side.cuda_stream)
        with torch.cuda.stream(side):
            run()
        torch.cuda.synchronize()
        free = tadm.tadm_pool_free_pages(w.pool)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for refused in (lambda: tadm.tadm_context_append(w.m, ctx, more, B, 70), lambda: tadm.tadm_pool_compact(w.pool)):
                with pytest.raises(tadm.TadmError, match="captured"):
                    refused()
            run()
        assert tadm.tadm_context_length(ctx) == 100 and tadm.tadm_pool_free_pages(w.pool) == free
        for i in range(4):
            if i == 2:  # the pages of ctx move
                tadm.tadm_context_destroy(first)
                with torch.cuda.stream(side):
                    tadm.tadm_pool_compact(w.pool)
            with torch.cuda.stream(side):
                logits.zero_()
                g.replay()
            torch.cuda.synchronize()
            assert torch.equal(logits, want), i
        tadm.tadm_set_stream(w.m, back.cuda_stream)
        tadm.tadm_cache_destroy(cache)
        tadm.tadm_context_destroy(ctx)
