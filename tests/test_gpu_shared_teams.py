"""Attention by plans whose blocks share several heads out over their waves, on the GPU: every number of heads, width and
head width that the plan may choose, and splits on either side, each shown to be reached by the plan's own items.

The plan gives a block 4 heads from 1 024 units (K/V heads x rows with tokens x tiles of columns) on where the K/V heads are a
multiple of 4, and 2 from 512 on where they are even."""
import numpy as np
import pytest
import torch

from test_gpu_pages_shared import check, shared_work, spread

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def mixed(rows, most, seed):
    """Lengths of rows: none, inside pages, at their ends."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, most + 1, size=rows)
    lens[::7] = lens[::7] // 64 * 64
    lens[3] = 0
    return lens.tolist()


TEAMS = [
    # K/V heads, queries each, head width, rows, tokens of a row at most, teams, width
    (16, 1, 64, 32, 1, 2, 16),
    (16, 1, 128, 32, 1, 2, 16),
    (16, 2, 64, 48, 3, 2, 16),
    (16, 2, 128, 63, 3, 2, 16),
    (6, 1, 64, 171, 1, 2, 16),     # even heads that are no multiple of 4
    (6, 2, 128, 171, 9, 2, 32),
    (8, 2, 64, 64, 10, 2, 32),
    (8, 2, 128, 64, 16, 2, 32),
    (16, 1, 64, 64, 5, 4, 16),
    (16, 1, 128, 64, 16, 4, 16),
    (16, 2, 64, 64, 12, 4, 32),
    (16, 4, 128, 64, 8, 4, 32),
    (4, 1, 64, 256, 2, 4, 16),     # more rows than a wave plans
    (4, 3, 128, 256, 6, 4, 32),
    (3, 1, 64, 342, 1, 1, 16),     # odd heads: each by itself
    (16, 1, 64, 31, 1, 1, 16),     # 496 units
    (8, 1, 64, 70, 33, 1, 64),     # wider: each by itself
]


@pytest.mark.parametrize("case", range(len(TEAMS)))
@pytest.mark.parametrize("shared", [0, 6])
def test_heads_shared_out_over_the_waves(case, shared):
    Hkv, G, dh, rows, n, teams, width = TEAMS[case]
    rng = np.random.default_rng(case)
    news = rng.integers(1, n + 1, size=rows)
    news[rows // 2] = n
    lens = [64 * shared + x for x in mixed(rows, 200, case)]
    plans = []
    check("bf16", G * Hkv, Hkv, dh, [(shared, lens)], news.tolist(), 500 + case, seen=plans, windowed=case % 3 != 2)
    _, items = shared_work(plans[0])
    own = items[items[:, 9] > 0]
    assert (own[:, 11] == teams).all() and (own[:, 4] == width).all()
    if teams > 1:
        assert len(own) == rows * Hkv // teams * -(-G * n // width)


def splits(items):
    """Items of a K/V head and tile of columns of a row or a group, at most."""
    _, counts = np.unique(items[:, [0, 1, 2, 3]], axis=0, return_counts=True)
    return int(counts.max()) if len(counts) else 0


SPLITS = [
    # dtype, H, Hkv, dh, prompts, tokens; whether a row's own keys, and shared pages, are split
    ("f32", 4, 4, 16, [(60, spread(3840, 16))], [1] * 16, None, True),
    ("f32", 2, 1, 20, [(0, [6000, 3000])], [2, 1], True, None),
    ("bf16", 32, 16, 128, [(130, spread(8320, 16, 31))], [1] * 16, None, True),
    ("bf16", 4, 4, 64, [(64, [4096 + 4000 + 64 * i for i in range(40)])], [1] * 40, None, None),
    ("bf16", 2, 2, 128, [(200, spread(18700, 16, 9))], [1] * 16, True, True),
    ("bf16", 4, 2, 128, [(0, [4500, 4480])], [3, 20], True, None),
    ("bf16", 2, 2, 128, [(0, [4500, 4480])], [130, 200], True, None),
    ("bf16", 2, 2, 64, [(0, [5000, 100])], [40, 64], True, None),
]


@pytest.mark.parametrize("case", range(len(SPLITS)))
def test_splits_on_either_side(case):
    dtype, H, Hkv, dh, prompts, news, own_split, shared_split = SPLITS[case]
    plans = []
    check(dtype, H, Hkv, dh, prompts, news, 700 + case, seen=plans)
    _, items = shared_work(plans[0])
    own, shared = splits(items[items[:, 9] > 0]), splits(items[items[:, 9] == 0])
    print(f"own splits {own}, shared {shared}")
    if own_split is not None:
        assert own > 1
    if shared_split is not None:
        assert shared > 1
