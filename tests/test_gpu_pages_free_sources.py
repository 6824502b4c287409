"""Forks of rows that name pages which are free (a state that a freed row's leftovers or a wrong count make): reported, not shared and
not given twice, and the same every time, in either form of the kernels."""
import copy

import pytest
import torch

from paper_2407_00079_amd import binding as B
from pages_util import BAD_ID, State
from test_gpu_pages import DEV, Device, ints

pytestmark = pytest.mark.gpu


def forked(state, src, dst):
    """What a fork makes of such a state: entries are copied as they are, counts of free pages stay, free pages go out lowest first."""
    s, free, moves, flags = copy.deepcopy(state), state.free_pages(), [], 0
    for a, b in zip(src, dst):
        n = s.lens[a]
        for j in range(n // s.page):
            page = state.tables[a][j]
            s.tables[b][j] = page
            if state.inside(page) and state.counts[page]:
                s.counts[page] += 1
            else:
                flags |= BAD_ID
        if n % s.page:
            j, new = n // s.page, free.pop(0)
            page = state.tables[a][j]
            if not (state.inside(page) and state.counts[page]):
                flags |= BAD_ID
            s.tables[b][j] = new
            s.counts[new] = 1
            moves.append([-1 if state.inside(page) and not state.counts[page] else page, new])
        s.lens[b] = n
    return s, moves, [len(moves), flags, len(free), len(moves)]


def check(state, src, dst):
    for _ in range(3):
        d = Device(copy.deepcopy(state))
        got = ints([[7, 7]] * len(src))
        B.mc_kv_pages_fork(d.counts, d.tables, state.page, d.lens, ints(src), ints(dst), got, d.report, d.ws)
        d.plain, moves, report = forked(state, src, dst)
        d.same(report, moves, got)
    return got, report


@pytest.mark.parametrize("pages,wide", [(40, 6), (20000, 2000)])
def test_sources_that_name_free_pages(pages, wide):
    tables = [[-5] * wide for _ in range(9)]
    # pages 0 and up are given out to the forks; 30 is free and stays so; `pages` is outside of the pool
    tables[0][:4], tables[1][:3], tables[2][:3], tables[3][:2] = [10, 0, 30, 11], [0, 1, 12], [13, 13, 30], [pages, 1]
    counts = [0] * pages
    for page in (10, 11, 12, 13):
        counts[page] = 1
    counts[13] = 2
    state = State(counts, tables, 16, [60, 48, 40, 20, 0, 0, 0, 0, 0])
    for src, dst in (([0], [4]), ([1], [5]), ([2], [4]), ([3], [8]), ([0, 1, 2, 3, 0], [4, 5, 6, 7, 8])):
        got, report = check(state, src, dst)
        assert report[1] == BAD_ID
        pool = (torch.arange(pages * 16, device=DEV) % 251).to(torch.uint8).reshape(pages, 16)
        want = pool.clone()
        for s, t in got[: report[0]].tolist():
            if 0 <= s < pages:
                want[t] = pool[s]
        B.mc_kv_copy_pages([pool], [pool.clone()], pages, 16, got)
        assert torch.equal(pool, want)


@pytest.mark.parametrize("pages,wide,n", [(600, 4, 90), (16384, 4, 90), (9000, 400, 200), (40000, 30, 300)])
def test_many_forks_over_free_pages(pages, wide, n):
    """Every other page of the sources is free, and as many pages are given out as there are forks, low ones first."""
    rows = 3 + n
    tables = [[-5] * wide for _ in range(rows)]
    for r in range(3):
        tables[r] = [(r * wide + j) * 2 % pages for j in range(wide)]
    counts = [0] * pages
    for r in range(3):
        for j in range(0, wide, 2):
            counts[tables[r][j]] += 1
    state = State(counts, tables, 16, [wide * 16 - 9, wide * 16, wide * 16 - 1] + [0] * n)
    _, report = check(state, [i % 3 for i in range(n)], list(range(3, rows)))
    assert report[0] > n // 2 and report[1] == BAD_ID
