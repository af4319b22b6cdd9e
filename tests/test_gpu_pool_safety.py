"""What a page pool and its contexts must not do to one another, and the calls that they refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_pooled import World  # noqa: E402


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
