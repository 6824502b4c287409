"""Lists of moves that are not full and come without a count: the unused entries behind the moves are passed over."""
import copy

import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from pages_util import State, random_state
from test_gpu_pages import Device, ints, pools

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("unused", [0, 1, 2, 61])
def test_entries_and_counts_follow_the_moves_before_them(unused):
    counts = [0] * 16
    for page in (0, 10, 12, 15):
        counts[page] = 1
    d = Device(State(counts, [[10, 0, 12], [15, -1, 16], [12, 9, 9]], 16, [48, 40, 0]))
    moves = [[10, 1], [12, 2]]
    B.mc_kv_pages_remap(d.counts, d.tables, 16, d.lens, ints(moves + [[-1, -1]] * unused))
    d.plain.remap(moves)
    d.same([9, 9, 9, 9])


def test_a_list_without_moves():
    d = Device(State([1, 0, 1, 0], [[2, 0], [-1, 9]], 16, [32, 32]))
    B.mc_kv_pages_remap(d.counts, d.tables, 16, d.lens, ints([[-1, -1]] * 5))
    d.same([9, 9, 9, 9])


@pytest.mark.parametrize("pages,rows,wide,fill", [(300, 33, 20, 0.6), (16384, 60, 200, 0.5), (20000, 300, 60, 0.5)])
@pytest.mark.parametrize("room", ["more than moves", "one more", "as many", "fewer"])
def test_a_compaction_whose_report_is_not_read(pages, rows, wide, fill, room):
    d = Device(random_state(np.random.default_rng(pages), pages, rows, wide, 16, fill))
    every, _ = copy.deepcopy(d.plain).compact(pages)
    most = {"more than moves": pages, "one more": len(every) + 1, "as many": len(every), "fewer": len(every) // 2}[room]
    listed, k, v = ints([[7, 7]] * most), pools(2, pages, 64, 1), pools(2, pages, 64, 2)
    want = [x.clone() for x in k + v]
    B.mc_kv_pages_compact(d.counts, listed, d.report, d.ws)
    B.mc_kv_copy_pages(k, v, pages, 64, listed)
    B.mc_kv_pages_remap(d.counts, d.tables, 16, d.lens, listed)
    moves, report = d.plain.compact(most)
    d.plain.remap(moves)
    assert moves and listed.tolist() == moves + [[-1, -1]] * (most - len(moves))
    d.same(report)
    for s, t in moves:
        for x in want:
            x[t] = x[s]
    assert all(torch.equal(a, b) for a, b in zip(k + v, want))
