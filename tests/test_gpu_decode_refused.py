"""A captured decode step whose growth is refused: nothing is written, and the step goes on once there are pages again."""
import math

import pytest
import torch

from paper_2407_00079_amd import binding as B
from decode_util import assert_near, reference
from test_gpu_pages import DEV, ints

pytestmark = pytest.mark.gpu
PAGE, HQ, HKV, D, LAYERS, PAGES, WIDE = 16, 8, 2, 128, 2, 7, 3


class Serving:
    """Three rows in use, one of them a fork that shares its first page with row 0, one empty row; all lengths at a page's end or before it."""

    def __init__(self):
        torch.manual_seed(3)
        self.p, self.rope = B.attn_params(HQ, HKV, D, PAGE, PAGES, "bf16"), B.rope_params(D, B.MC_ROPE_HALF)
        self.k, self.v = ([torch.randn((PAGES, HKV, PAGE, D), device=DEV).to(torch.bfloat16) for _ in range(LAYERS)] for _ in range(2))
        self.tables, self.lens = ints([[0, 1, 9], [0, 9, 9], [2, 3, 4], [9, 9, 9]]), ints([30, 16, 47, 0])
        self.counts, self.report = ints([2, 1, 1, 1, 1, 1, 1]), ints([9] * 4)                 # 5 and 6 are other users': none is free
        self.add, self.step_lens = ints([7] * 4), ints([7] * 4)
        self.ws = torch.empty(B.mc_kv_pages_workspace_bytes(PAGES, 4), dtype=torch.uint8, device=DEV)
        self.attn_ws = torch.empty(B.mc_decode_attn_workspace_bytes(self.p, 4), dtype=torch.uint8, device=DEV)
        self.new = torch.randn((LAYERS, 4, (HQ + 2 * HKV) * D), device=DEV).to(torch.bfloat16)
        self.q_rot, self.outs = (torch.full((LAYERS, 4, HQ, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def step(self):
        self.add.copy_(self.lens > 0)                         # a token for each row in use
        B.mc_kv_pages_grow(self.counts, self.tables, PAGE, self.lens, self.add, self.report, self.ws)
        torch.mul(self.lens, self.report[1:2] == 0, out=self.step_lens)     # growth refused: every row is a padding row
        for layer in range(LAYERS):
            q, k, v = self.new[layer].split((HQ * D, HKV * D, HKV * D), dim=1)
            B.mc_kv_rope_append_decode(self.p, self.rope, q, k, v, None, None, self.q_rot[layer], self.k[layer], self.v[layer], self.tables,
                                       self.step_lens)
            B.mc_decode_attn_paged(self.p, self.q_rot[layer], self.k[layer], self.v[layer], self.tables, self.step_lens, self.outs[layer], None,
                                   self.attn_ws)

    def captured(self):
        self.step()                                           # (refused, as the first replays are)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        return graph

    def state(self):
        return [x.clone() for x in (self.counts, self.tables, self.lens, *self.k, *self.v)]


def test_refused_for_want_of_pages():
    s = Serving()
    before = s.state()
    graph = s.captured()
    for _ in range(3):
        s.outs.fill_(math.nan)
        graph.replay()
        assert s.report.tolist() == [0, B.MC_PAGES_SHORT, 0, 1]
        assert all(torch.equal(a, b) for a, b in zip(before, s.state())) and bool((s.outs == 0).all())
        torch.cuda.synchronize()
    s.counts[6] = 0                                           # a page is given back
    graph.replay()
    assert s.report.tolist() == [1, 0, 0, 1] and s.lens.tolist() == [31, 17, 48, 0] and s.tables[1].tolist() == [0, 6, 9]
    for layer in range(LAYERS):
        v = s.new[layer, :, (HQ + HKV) * D:].reshape(4, HKV, D)
        assert torch.equal(s.v[layer][1, :, 14], v[0]) and torch.equal(s.v[layer][6, :, 0], v[1]) and torch.equal(s.v[layer][4, :, 15], v[2])
        out, _, off, _ = reference(s.q_rot[layer], s.k[layer], s.v[layer], s.tables, [31, 17, 48, 0], 1 / math.sqrt(D))
        assert_near(s.outs[layer], out, off, f"layer {layer}")
        for x, old in ((s.k[layer], before[3 + layer]), (s.v[layer], before[3 + LAYERS + layer])):       # and nothing else was
            same = (x == old).all(-1)
            same[1, :, 14] = same[6, :, 0] = same[4, :, 15] = True
            assert bool(same.all())


def test_refused_at_the_end_of_a_table():
    s = Serving()
    s.lens[2] = 48
    s.counts[5:] = 0
    before = s.state()
    graph = s.captured()
    for _ in range(3):
        s.outs.fill_(math.nan)
        graph.replay()
        assert s.report.tolist()[:2] == [0, B.MC_PAGES_BAD_ROW]
        assert all(torch.equal(a, b) for a, b in zip(before, s.state())) and bool((s.outs == 0).all())
        torch.cuda.synchronize()
    B.mc_kv_pages_free(s.counts, s.tables, PAGE, s.lens, ints([2]), s.report)
    graph.replay()
    assert s.report.tolist()[1] == 0 and s.lens.tolist() == [31, 17, 0, 0]
    for layer in range(LAYERS):
        out, _, off, _ = reference(s.q_rot[layer], s.k[layer], s.v[layer], s.tables, [31, 17, 0, 0], 1 / math.sqrt(D))
        assert_near(s.outs[layer], out, off, f"layer {layer}")
