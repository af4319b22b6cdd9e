"""Page tables kept on the device against the oracle: whole numbers, compared exactly."""
import copy

import numpy as np
import pytest
import torch

import synth
from oracle import pages as P

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def m():
    m = tadm.tadm_model_create(tadm.make_config(synth.get_config("tiny"), max_batch=4, max_seq=256))
    tadm.tadm_set_stream(m, torch.cuda.current_stream().cuda_stream)
    yield m
    tadm.tadm_model_destroy(m)


class Book:
    """The same stack and tables on the GPU and for the oracle."""

    def __init__(self, rng, lens, max_pages, free, spare=0):
        held = [P._up(x) for x in lens]
        self.size = sum(held) + free + spare
        ids = rng.permutation(self.size).tolist()
        self.table = [[ids.pop() for _ in range(h)] + [-1] * (max_pages - h) for h in held]
        self.ids, self.free, self.lens = [ids.pop() for _ in range(free)], free, list(lens)
        self.ids += [-7] * (self.size - free)
        self.ids_dev, self.state, self.table_dev = i32(self.ids), i32([free, 0, 0, 0]), i32(self.table)
        self.stack = tadm.page_stack(self.ids_dev, self.state)

    def rows(self, most, lens, news):
        return tadm.page_rows(self.table_dev, most, lens, news)

    def same(self):
        torch.cuda.synchronize()
        assert self.state.tolist() == [self.free, 0, 0, 0]
        assert self.ids_dev[:self.free].tolist() == self.ids[:self.free]
        assert self.table_dev.tolist() == self.table


CASES = [
    # lengths, new tokens, free pages, spare entries of a row's table
    ([0], [1], 1, 0),
    ([63, 64, 65, 0], [1, 1, 1, 1], 4, 1),
    ([10, 200, 64], [0, 0, 0], 3, 0),
    ([100, 7, 333, 64], [64, 500, 1, 128], 5, 0),         # the second row does not get its pages, the third needs none
    ([100, 7, 333, 64], [64, 500, 64, 128], 2, 2),
    ([5, 5], [60, 60], 0, 3),                             # an empty stack, rows that need one page each
    ([128] * 300, [1] * 300, 299, 0),                     # more rows than threads; the last has to wait
    ([0, 1, 64, 4000], [4096, 2047, 2049, 6000], 1000, 1),  # windows of several chunks
]


@pytest.mark.parametrize("lens, news, free, more", CASES)
@pytest.mark.parametrize("want_slots", [True, False])
def test_assign_and_release(m, lens, news, free, more, want_slots):
    rng = np.random.default_rng(len(lens) + free)
    B, n = len(lens), max(max(news), 1)
    mp = max(P._up(a + b) for a, b in zip(lens, news)) + more
    book = Book(rng, lens, mp, free, spare=3)
    ln, nw, granted = i32(lens), i32(news), torch.full((B,), 99, dtype=torch.int32, device="cuda")
    slots = torch.full((B, n), 99, dtype=torch.int64, device="cuda") if want_slots else None
    ref_granted, ref_slots, book.free = P.assign(book.table, lens, news, book.ids, book.free, book.size)
    tadm.tadm_pages_assign(m, book.stack, book.rows(mp * 64, ln, nw), n, granted, slots)
    book.same()
    assert granted.tolist() == ref_granted
    if want_slots:
        assert slots.tolist() == [s + [-1] * (n - len(s)) for s in ref_slots]
    # half of the tokens come back, then the others
    for keep, gone in (([a + g // 2 for a, g in zip(lens, ref_granted)], [g - g // 2 for g in ref_granted]),
                       (lens, [g // 2 for g in ref_granted])):
        book.free = P.release(book.table, keep, gone, book.ids, book.free, book.size)
        tadm.tadm_pages_release(m, book.stack, book.rows(mp * 64, i32(keep), i32(gone)), n)
        book.same()


def test_lengths_of_the_host(m):
    """Without device lengths every row has the same: len and n."""
    book = Book(np.random.default_rng(1), [70, 70, 70], 4, 5)
    granted = i32([9, 9, 9])
    rows = tadm.page_rows(book.table_dev, 70)
    ref, _, book.free = P.assign(book.table, [70] * 3, [130] * 3, book.ids, book.free, book.size)
    tadm.tadm_pages_assign(m, book.stack, rows, 130, granted)
    book.same()
    assert granted.tolist() == ref == [130, 130, 0]
    book.free = P.release(book.table, [70] * 3, ref, book.ids, book.free, book.size)
    tadm.tadm_pages_release(m, book.stack, tadm.page_rows(book.table_dev, 70, None, granted), 130)
    book.same()


def test_lengths_past_their_bounds(m):
    """Device lengths are cut to [0, len] and [0, n]; a row past its table gets nothing and gives nothing back."""
    book = Book(np.random.default_rng(2), [64, 0, 64], 2, 8)
    granted, slots = i32([0, 0, 0]), torch.zeros(3, 100, dtype=torch.int64, device="cuda")
    tadm.tadm_pages_assign(m, book.stack, book.rows(64, i32([64, -5, 900]), i32([100, 1000, -3])), 100, granted, slots)
    ref, ref_slots, book.free = P.assign(book.table, [64, 0, 64], [100, 100, 0], book.ids, 8, book.size)
    assert granted.tolist() == ref == [0, 100, 0]
    assert slots.tolist() == [s + [-1] * (100 - len(s)) for s in ref_slots]
    book.same()
    tadm.tadm_pages_release(m, book.stack, book.rows(64, i32([64, -5, 900]), i32([100, 1000, -3])), 100)
    book.free = P.release(book.table, [64, 0, 64], [100, 100, 0], book.ids, book.free, book.size)
    book.same()


def test_many_rows_and_entries_that_name_no_page(m):
    """4 096 rows (the most of a call); absent and foreign entries become -1 and nothing else."""
    rng = np.random.default_rng(3)
    lens, news = rng.integers(0, 300, size=4096).tolist(), rng.integers(0, 150, size=4096).tolist()
    mp = P._up(450)
    book = Book(rng, lens, mp, 6000)
    n = 150
    granted = torch.zeros(4096, dtype=torch.int32, device="cuda")
    slots = torch.zeros(4096, n, dtype=torch.int64, device="cuda")
    ref, ref_slots, book.free = P.assign(book.table, lens, news, book.ids, book.free, book.size)
    tadm.tadm_pages_assign(m, book.stack, book.rows(mp * 64, i32(lens), i32(news)), n, granted, slots)
    book.same()
    assert granted.tolist() == ref and slots.tolist() == [s + [-1] * (n - len(s)) for s in ref_slots]
    for b in range(0, 4096, 5):
        e = P._up(lens[b])
        if P._up(lens[b] + ref[b]) > e:
            book.table[b][e] = (-1, book.size, 2147483647, -2147483648)[b % 4]
    book.table_dev.copy_(i32(book.table))
    book.free = P.release(book.table, lens, ref, book.ids, book.free, book.size)
    tadm.tadm_pages_release(m, book.stack, book.rows(mp * 64, i32(lens), granted), n)
    book.same()


def test_a_page_that_comes_back_twice_stays_inside_the_stack(m):
    ids, state = i32([0, 1, 2, 3]), i32([4, 0, 0, 0])
    guard = torch.full((8,), 55, dtype=torch.int32, device="cuda")
    table = i32([[1, 2], [1, 2]])
    tadm.tadm_pages_release(m, tadm.page_stack(ids, state), tadm.page_rows(table, 128, i32([0, 0]), i32([128, 128])), 128)
    torch.cuda.synchronize()
    assert ids.tolist() == [0, 1, 2, 3] and state.tolist() == [4, 0, 0, 0] and guard.eq(55).all() and table.eq(-1).all()


@pytest.mark.parametrize("count", [-3, 1000])
def test_a_count_outside_the_stack_is_cut(m, count):
    ids, state, table = i32([3, 1, 0, 2]), i32([count, 0, 0, 0]), i32([[-1, -1], [-1, -1]])
    granted = i32([0, 0])
    tadm.tadm_pages_assign(m, tadm.page_stack(ids, state), tadm.page_rows(table, 0), 100, granted)
    torch.cuda.synchronize()
    free = min(max(count, 0), 4)
    assert granted.tolist() == [100 if free >= 2 else 0, 100 if free >= 4 else 0]
    assert table.tolist() == ([[2, 0], [1, 3]] if free == 4 else [[-1, -1]] * 2) and state.tolist()[0] == 0


def test_captured_turns_follow_the_lengths(m):
    """A captured assign and release serve the lengths of each replay, with eager work of the program in between."""
    rng = np.random.default_rng(4)
    lens = [100, 64, 0, 700]
    book = Book(rng, lens, 30, 40)
    ln, nw, granted = i32(lens), i32([0] * 4), i32([0] * 4)
    slots = torch.zeros(4, 512, dtype=torch.int64, device="cuda")
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    take, give = book.rows(1000, ln, nw), book.rows(1000, ln, granted)
    side.wait_stream(main)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        tadm.tadm_set_stream(m, side.cuda_stream)
        try:
            with torch.cuda.graph(graph, stream=side):
                tadm.tadm_pages_assign(m, book.stack, take, 512, granted, slots)
                tadm.tadm_pages_release(m, book.stack, give, 512)
        finally:
            tadm.tadm_set_stream(m, main.cuda_stream)
    main.wait_stream(side)
    for news in ([1, 1, 1, 1], [512, 500, 300, 0], [511, 512, 512, 512], [0, 0, 0, 0], [27, 1, 64, 5]):
        nw.copy_(i32(news))
        before = copy.deepcopy(book.table)
        ref, ref_slots, book.free = P.assign(book.table, lens, news, book.ids, book.free, book.size)
        book.free = P.release(book.table, lens, ref, book.ids, book.free, book.size)
        graph.replay()
        book.same()
        assert book.table == before and granted.tolist() == ref
        assert slots.tolist() == [s + [-1] * (512 - len(s)) for s in ref_slots]
        torch.cuda.synchronize()


def test_rows_of_a_pooled_context_are_refused():
    cfg = synth.get_config("tiny")
    m = tadm.load_model(cfg, [t.cuda() for t in synth.make_weights(cfg)], max_batch=2, max_seq=256,
                        stream=torch.cuda.current_stream().cuda_stream)
    pool = tadm.tadm_pool_create(m, 8)
    ctx = tadm.tadm_context_create_pooled(m, pool, 2, 256)
    try:
        stack, granted = tadm.page_stack(i32([0, 1]), i32([2, 0, 0, 0])), i32([0, 0])
        for what in (lambda r: tadm.tadm_pages_assign(m, stack, r, 1, granted), lambda r: tadm.tadm_pages_release(m, stack, r, 1)):
            with pytest.raises(tadm.TadmError) as e:
                what(tadm.tadm_context_rows(ctx))
            assert e.value.status == tadm.TADM_ERR_STATE
    finally:
        tadm.tadm_context_destroy(ctx)
        tadm.tadm_pool_destroy(pool)
        tadm.tadm_model_destroy(m)
