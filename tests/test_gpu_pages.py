"""Rows forked, grown and freed, pools compacted, pages copied: integers and bytes, equal to the plain form's."""
import copy

import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from pages_util import BAD_ID, BAD_ROW, SHORT, State, random_state

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


class Device:
    """A state on the GPU beside its plain form; every call is made on both and compared."""

    def __init__(self, plain):
        self.plain = plain
        self.counts, self.lens = ints(plain.counts), ints(plain.lens)
        self.tables = ints(plain.tables).reshape(len(plain.lens), plain.wide)
        self.ws = torch.full((B.mc_kv_pages_workspace_bytes(len(plain.counts), len(plain.lens)),), 255, dtype=torch.uint8, device=DEV)
        self.report = ints([9, 9, 9, 9])

    def same(self, report, moves=None, got=None):
        assert self.report.tolist() == report
        if moves is not None:
            assert got.tolist() == moves + [[-1, -1]] * (got.shape[0] - len(moves))
        assert self.counts.tolist() == self.plain.counts and self.lens.tolist() == self.plain.lens
        assert self.tables.tolist() == self.plain.tables

    def fork(self, src, dst):
        got = ints([[7, 7]] * len(src))
        B.mc_kv_pages_fork(self.counts, self.tables, self.plain.page, self.lens, ints(src), ints(dst), got, self.report, self.ws)
        moves, report = self.plain.fork(src, dst)
        self.same(report, moves, got)
        return got, report

    def grow(self, add):
        B.mc_kv_pages_grow(self.counts, self.tables, self.plain.page, self.lens, ints(add), self.report, self.ws)
        report = self.plain.grow(add)
        self.same(report)
        return report

    def free(self, rows):
        B.mc_kv_pages_free(self.counts, self.tables, self.plain.page, self.lens, ints(rows), self.report)
        report = self.plain.free(rows)
        self.same(report)
        return report

    def compact(self, most):
        got = ints([[7, 7]] * most)
        B.mc_kv_pages_compact(self.counts, got, self.report, self.ws)
        moves, report = self.plain.compact(most)
        self.same(report, moves, got)
        count = self.report[:1].clone()
        B.mc_kv_pages_remap(self.counts, self.tables, self.plain.page, self.lens, got, count)
        self.plain.remap(moves)
        self.same(report)
        return got, report


# pages, rows, columns, tokens a page, filled
SIZES = [(1, 1, 1, 16, 1.0), (40, 5, 6, 16, 0.5), (300, 33, 20, 16, 0.6), (4096, 40, 90, 16, 0.5), (4097, 70, 90, 1, 0.4), (9000, 200, 60, 7, 0.7),
         (16384, 60, 200, 16, 0.5), (16385, 60, 200, 16, 0.5), (9000, 400, 130, 16, 0.8), (20000, 1300, 30, 16, 0.5), (40000, 300, 220, 16, 0.6)]


@pytest.mark.parametrize("pages,rows,wide,page,fill", SIZES)
@pytest.mark.parametrize("seed", range(3))
def test_a_life_of_calls(pages, rows, wide, page, fill, seed):
    """Forks, growth, rows freed and pools compacted in turn, each step equal to the plain form, refusals among them."""
    rng = np.random.default_rng(seed * 1000 + pages)
    d = Device(random_state(rng, pages, rows, wide, page, fill))
    for step in range(4):
        empty = [r for r, n in enumerate(d.plain.lens) if n == 0]
        n = int(rng.integers(0, len(empty) + 1)) if empty else 0
        if n:
            dst = [int(x) for x in rng.permutation(empty)[:n]]
            d.fork([int(x) for x in rng.integers(0, rows, n)], dst)
        room = [d.plain.wide * page - n for n in d.plain.lens]
        d.grow([int(rng.integers(-2, min(x, 40) + 1)) if rng.random() < 0.6 else 0 for x in room])
        d.free([int(x) for x in rng.integers(0, rows, int(rng.integers(1, rows + 1)))])       # rows twice, empty rows among them
        d.compact(int(rng.integers(1, pages + 3)))


def test_pages_are_given_in_list_and_row_order():
    d = Device(State([0, 1, 0, 0, 1, 0, 0, 0], [[1, 4, 9], [9, 9, 9], [9, 9, 9], [9, 9, 9]], 16, [20, 0, 0, 0]))
    got, report = d.fork([0, 0], [3, 1])
    assert got.tolist() == [[4, 0], [4, 2]] and report == [2, 0, 4, 2]
    assert d.grow([0, 13, 40, 0]) == [4, 0, 0, 4] and d.tables.tolist()[1:3] == [[1, 2, 3], [5, 6, 7]]


def test_too_few_pages_changes_nothing():
    d = Device(State([1, 1, 0], [[0, 1], [9, 9], [9, 9]], 16, [17, 0, 0]))
    assert d.fork([0, 0], [1, 2])[1] == [0, SHORT, 1, 2]
    assert d.grow([0, 16, 17]) == [0, SHORT, 1, 3]
    assert d.grow([15, 0, 16]) == [1, 0, 0, 1]
    assert d.grow([0, 1, 0]) == [0, SHORT, 0, 1]


def test_what_is_not_valid_is_refused_on_the_device():
    plain = State([1, 1, 0, 0, 0, 0, 0, 0], [[0, 1], [9, 9], [9, 9], [9, 9]], 16, [17, 0, 0, 0])
    for src, dst in (([4], [1]), ([-1], [1]), ([0], [4]), ([0], [-1]), ([0], [0]), ([1], [0]), ([0, 9], [1, 2])):
        assert Device(copy.deepcopy(plain)).fork(src, dst)[1][:2] == [0, BAD_ROW]
    d = Device(copy.deepcopy(plain))                          # a row made twice: which entry counts is not said
    got = ints([[7, 7]] * 3)
    B.mc_kv_pages_fork(d.counts, d.tables, 16, d.lens, ints([0, 0, 0]), ints([1, 2, 1]), got, d.report, d.ws)
    assert d.report.tolist()[:3] == [0, BAD_ROW, 6] and got.tolist() == [[-1, -1]] * 3
    assert d.counts.tolist() == plain.counts and d.lens.tolist() == plain.lens and d.tables.tolist() == plain.tables
    assert Device(copy.deepcopy(plain)).grow([16, 0, 0, 0])[:2] == [0, BAD_ROW]
    assert Device(copy.deepcopy(plain)).grow([2 ** 31 - 1, 0, 0, 0])[:2] == [0, BAD_ROW]
    for lens in ([40, 0, 0, 0], [-3, 0, 0, 0]):
        bad = copy.deepcopy(plain)
        bad.lens = lens
        assert Device(copy.deepcopy(bad)).fork([0], [1])[1][:2] == [0, BAD_ROW]
        assert Device(copy.deepcopy(bad)).grow([1, 5, 0, 0])[:2] == [0, BAD_ROW]
        assert Device(copy.deepcopy(bad)).grow([0, 5, 0, 0])[:2] == [1, 0]
        assert Device(copy.deepcopy(bad)).free([0])[:2] == [0, BAD_ROW]
    assert Device(copy.deepcopy(plain)).free([4, 0, -1, 0])[:2] == [2, BAD_ROW]
    bad = copy.deepcopy(plain)
    bad.counts = [1, 0, 0, 0, 0, 0, 0, 0]                     # page 1 was free already
    assert Device(bad).free([0])[:2] == [1, BAD_ID]
    bad = copy.deepcopy(plain)
    bad.tables[0] = [8, 1]                                    # no page of the pool
    assert Device(copy.deepcopy(bad)).free([0])[:2] == [1, BAD_ID]
    assert Device(bad).fork([0], [1])[1][:2] == [1, BAD_ID]


@pytest.mark.parametrize("pages,wide", [(40, 4), (20000, 2000)])
def test_pages_that_are_none(pages, wide):
    """Entries outside the pool, among full pages and as a row's last page: reported, never followed, in either form of the kernels."""
    tables = [[-5] * wide for _ in range(6)]
    tables[0][:3], tables[1][:3], tables[2][:2] = [3, pages, 5], [7, 8, 2 ** 31 - 1], [-1, 9]
    counts = [0] * pages
    for page in (3, 5, 7, 8, 9):
        counts[page] = 1
    state = State(counts, tables, 16, [48, 40, 32, 0, 0, 0])
    assert Device(copy.deepcopy(state)).fork([0, 1, 2], [3, 4, 5])[1] == [1, BAD_ID, pages - 6, 1]
    d = Device(copy.deepcopy(state))
    moves, report = d.fork([1], [5])
    assert report[:2] == [1, BAD_ID] and moves.tolist() == [[2 ** 31 - 1, 0]]
    pool = (torch.arange(pages * 16, device=DEV) % 251).to(torch.uint8)
    before = pool.clone()
    B.mc_kv_copy_pages([pool], [pool], pages, 16, moves, d.report[:1])
    assert torch.equal(pool, before)
    assert Device(copy.deepcopy(state)).free([0, 1, 2])[:2] == [5, BAD_ID]
    assert Device(copy.deepcopy(state)).grow([1, 0, 0, 20, 0, 0])[:2] == [3, 0]


def test_nothing_to_do():
    d = Device(random_state(np.random.default_rng(1), 50, 4, 5, 16, 0.5))
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    B.mc_kv_pages_fork(d.counts, d.tables, 16, d.lens, empty, empty, empty.reshape(0, 2), d.report, d.ws)
    B.mc_kv_pages_free(d.counts, d.tables, 16, d.lens, empty, d.report)
    B.mc_kv_pages_compact(d.counts, empty.reshape(0, 2), d.report, d.ws)
    B.mc_kv_pages_remap(d.counts, d.tables, 16, d.lens, empty.reshape(0, 2))
    B.mc_kv_copy_pages([], [], 50, 64, ints([[1, 2]]))
    d.same([9, 9, 9, 9])                                      # the report too is as it was
    full = Device(State([1] * 8192, [[0]], 16, [16]))
    assert full.compact(5)[1] == [0, 0, 0, 0]
    none = Device(State([0] * 8192, [[0]], 16, [0]))
    assert none.compact(5)[1] == [0, 0, 8192, 0]


def pools(layers, pages, page_bytes, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return [torch.randint(0, 256, (pages, page_bytes), dtype=torch.uint8, device=DEV, generator=gen) for _ in range(layers)]


@pytest.mark.parametrize("page_bytes", [16, 4096, 8192, 8208, 32768, 70000 // 16 * 16])
@pytest.mark.parametrize("layers,n", [(1, 1), (3, 50), (128, 2), (2, 333)])
def test_copied_pages(page_bytes, layers, n):
    pages = 2 * n + 5
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(n))[: 2 * n].to(torch.int32).reshape(2, n).t().contiguous()
    if n > 3:
        order[1, 0] = order[0, 0]                             # a page copied twice
        order[2], order[3] = torch.tensor([-1, -1]), torch.tensor([0, pages])                 # and moves that are none
        order[4:][order[4:, 1] == 0, 1] = -1
    moves = order.to(DEV)
    for count in (None, n // 2, 0, n + 7, -1):
        k, v = pools(layers, pages, page_bytes, 1), pools(layers, pages, page_bytes, 2)
        want = [x.clone() for x in k + v]
        used = n if count is None else max(0, min(n, count))
        for s, t in order[:used].tolist():
            if 0 <= s < pages and 0 <= t < pages:
                for x in want:
                    x[t] = x[s]
        B.mc_kv_copy_pages(k, v, pages, page_bytes, moves, None if count is None else ints([count]))
        assert all(torch.equal(a, b) for a, b in zip(k + v, want))


def test_copied_pages_past_32_bits_of_bytes():
    page_bytes, pages = 32768, 140000
    k, v = (torch.empty((pages, page_bytes), dtype=torch.uint8, device=DEV) for _ in range(2))
    for x, mark in ((k, 3), (v, 5)):
        x[pages - 2] = mark
        x[1] = mark + 1
    B.mc_kv_copy_pages([k], [v], pages, page_bytes, ints([[pages - 2, 0], [1, pages - 1]]))
    assert bool((k[0] == 3).all()) and bool((v[0] == 5).all()) and bool((k[pages - 1] == 4).all()) and bool((v[pages - 1] == 6).all())


def test_a_replayed_step():
    """Fork, copy, growth, free and compaction captured once: every replay does what the eager calls do to the same state."""
    rng = np.random.default_rng(5)
    plain = random_state(rng, 600, 24, 12, 16, 0.5)
    d = Device(plain)
    src = ints([r for r, n in enumerate(plain.lens) if n][:5])
    dst = ints([r for r, n in enumerate(plain.lens) if n == 0][:5])
    src = src[: dst.shape[0]]
    dst = dst[: src.shape[0]]
    add = ints([3 if r in dst.tolist() else 0 for r in range(24)])
    k, v = pools(2, 600, 4096, 8), pools(2, 600, 4096, 9)
    start = [x.clone() for x in (d.counts, d.tables, d.lens, *k, *v)]
    state = [d.counts, d.tables, d.lens, *k, *v]
    moves, listed = ints([[0, 0]] * src.shape[0]), ints([[0, 0]] * 600)
    reports = [ints([0] * 4) for _ in range(4)]

    def step():
        B.mc_kv_pages_fork(d.counts, d.tables, 16, d.lens, src, dst, moves, reports[0], d.ws)
        B.mc_kv_copy_pages(k, v, 600, 4096, moves, reports[0])
        B.mc_kv_pages_grow(d.counts, d.tables, 16, d.lens, add, reports[1], d.ws)
        B.mc_kv_pages_free(d.counts, d.tables, 16, d.lens, src, reports[2])
        B.mc_kv_pages_compact(d.counts, listed, reports[3], d.ws)
        B.mc_kv_copy_pages(k, v, 600, 4096, listed, reports[3])
        B.mc_kv_pages_remap(d.counts, d.tables, 16, d.lens, listed, reports[3])

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (*state, moves, listed, *reports)]
    assert reports[0].tolist()[0] > 0 and reports[3].tolist()[0] > 0 and all(r.tolist()[1] == 0 for r in reports)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for to, x in zip(state, start):
            to.copy_(x)
        for x in (moves, listed, *reports):
            x.fill_(77)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((*state, moves, listed, *reports), want))
        torch.cuda.synchronize()
