"""Prompts, forks, captured decode steps, rows freed and the pool compacted, in the order a serving program makes the calls: two
layers, every row's attention checked at every step against the definition over that row's own history."""
import math

import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from gpu_util import TOL, check_close
from paper_2407_00079_amd import workloads as W
from rope_util import turned

pytestmark = pytest.mark.gpu
DEV, PAGE, LAYERS, HQ, HKV, D, ROTARY = "cuda:0", 16, 2, 8, 2, 128, 96


class History:
    """What the rows have seen, in 64 bits: rotated keys as the cache holds them (rounded to bf16) and values."""

    def __init__(self, rows, inv_freq, weights):
        self.k = [[[] for _ in range(rows)] for _ in range(LAYERS)]
        self.v = [[[] for _ in range(rows)] for _ in range(LAYERS)]
        self.inv_freq, self.weights = inv_freq, weights

    @staticmethod
    def rounded(x):
        return torch.from_numpy(x).to(torch.bfloat16).double().numpy()

    def turn(self, x, weight, pos):
        return self.rounded(turned(x.double().cpu().numpy(), weight, pos, self.inv_freq, ROTARY, False)[0])

    def add(self, layer, row, q, k, v):
        """New tokens of a row: their rotated queries."""
        pos = np.arange(len(self.k[layer][row]), len(self.k[layer][row]) + k.shape[0])
        self.k[layer][row] += list(self.turn(k.reshape(-1, HKV, D), self.weights[1], pos))
        self.v[layer][row] += list(v.double().cpu().numpy().reshape(-1, HKV, D))
        return self.turn(q.reshape(-1, HQ, D), self.weights[0], pos)

    def attend(self, layer, row, q, keys):
        """One query row [HQ, D] over the first `keys` keys."""
        k, v = np.stack(self.k[layer][row][:keys]), np.stack(self.v[layer][row][:keys])
        out = np.zeros((HQ, D))
        for h in range(HQ):
            s = k[:, h // (HQ // HKV)] @ q[h] / math.sqrt(D)
            p = np.exp(s - s.max())
            out[h] = p @ v[:, h // (HQ // HKV)] / p.sum()
        return out

    def fork(self, src, dst):
        for x in (self.k, self.v):
            for layer in range(LAYERS):
                x[layer][dst] = list(x[layer][src])

    def free(self, row):
        for x in (self.k, self.v):
            for layer in range(LAYERS):
                x[layer][row] = []


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def test_from_prompts_to_a_compacted_pool():
    torch.manual_seed(20)
    rows, wide, pages = 6, 14, 64
    p, rope = B.attn_params(HQ, HKV, D, PAGE, pages, "bf16"), B.rope_params(ROTARY, B.MC_ROPE_HALF)
    weights = [(1 + 0.2 * torch.randn(D, device=DEV)).to(torch.bfloat16) for _ in range(2)]
    past = History(rows, list(rope.inv_freq), [w.double().cpu().numpy() for w in weights])
    # NaN patterns everywhere: only the calls fill the pools
    k_pools, v_pools = ([torch.full((pages, HKV, PAGE, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(LAYERS)] for _ in range(2))
    counts, lens, tables = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV), ints([[0] * wide] * rows)
    counts[::3] = 1                                           # pages of other users
    others = int((counts > 0).sum())
    pages_ws = torch.empty(B.mc_kv_pages_workspace_bytes(pages, rows), dtype=torch.uint8, device=DEV)
    attn_ws = torch.empty(B.mc_decode_attn_workspace_bytes(p, rows), dtype=torch.uint8, device=DEV)
    report = ints([0] * 4)

    # prompts of rows 0 and 1
    prompt = [70, 37] + [0] * (rows - 2)
    B.mc_kv_pages_grow(counts, tables, PAGE, lens, ints(prompt), report, pages_ws)
    assert report.tolist()[:2] == [8, 0]
    total = sum(prompt)
    append_ws = torch.empty(B.mc_kv_append_workspace_bytes(rows), dtype=torch.uint8, device=DEV)
    prefill_ws = torch.empty(B.mc_prefill_attn_workspace_bytes(p, rows, total), dtype=torch.uint8, device=DEV)
    for layer in range(LAYERS):
        qkv = torch.randn((total, (HQ + 2 * HKV) * D), device=DEV).to(torch.bfloat16)
        q, k, v = qkv.split((HQ * D, HKV * D, HKV * D), dim=1)
        q_out, out = (torch.empty((total, HQ, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        B.mc_kv_rope_append_paged(p, rope, q, k, v, *weights, q_out, k_pools[layer], v_pools[layer], tables, [0] * rows, prompt, append_ws)
        B.mc_prefill_attn_paged(p, q_out, k_pools[layer], v_pools[layer], tables, [0] * rows, prompt, out, None, prefill_ws)
        at = 0
        for r, n in enumerate(prompt):
            turned_q = past.add(layer, r, q[at: at + n], k[at: at + n], v[at: at + n]) if n else []
            want = [past.attend(layer, r, turned_q[i], i + 1) for i in range(n)]
            if n:
                check_close(out[at: at + n].double().cpu().numpy(), np.stack(want), W.BF16, f"prompt {r} layer {layer}")
            at += n

    # two more answers to row 0's prompt
    moves = ints([[0, 0]] * 2)
    B.mc_kv_pages_fork(counts, tables, PAGE, lens, ints([0, 0]), ints([3, 4]), moves, report, pages_ws)
    B.mc_kv_copy_pages(k_pools, v_pools, pages, HKV * PAGE * D * 2, moves, report)
    assert report.tolist()[:2] == [2, 0]
    for r in (3, 4):
        past.fork(0, r)

    # a decode step, captured once; rows 2 and 5 are padding at first
    add, now = ints([1, 1, 0, 1, 1, 0]), torch.zeros((LAYERS, rows, (HQ + 2 * HKV) * D), dtype=torch.bfloat16, device=DEV)
    q_out, outs = torch.zeros((rows, HQ, D), dtype=torch.bfloat16, device=DEV), torch.zeros((LAYERS, rows, HQ, D), dtype=torch.bfloat16, device=DEV)

    def step():
        B.mc_kv_pages_grow(counts, tables, PAGE, lens, add, report, pages_ws)
        for layer in range(LAYERS):
            q, k, v = now[layer].split((HQ * D, HKV * D, HKV * D), dim=1)
            B.mc_kv_rope_append_decode(p, rope, q, k, v, *weights, q_out, k_pools[layer], v_pools[layer], tables, lens)
            B.mc_decode_attn_paged(p, q_out, k_pools[layer], v_pools[layer], tables, lens, outs[layer], None, attn_ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()

    def replay(times):
        for _ in range(times):
            now.copy_(torch.randn(now.shape, device=DEV))
            graph.replay()
            assert report.tolist()[1] == 0
            torch.cuda.synchronize()
            active = add.tolist()
            for layer in range(LAYERS):
                q, k, v = now[layer].split((HQ * D, HKV * D, HKV * D), dim=1)
                for r in range(rows):
                    if not active[r]:
                        assert bool((outs[layer, r] == 0).all())
                        continue
                    turned_q = past.add(layer, r, q[r: r + 1], k[r: r + 1], v[r: r + 1])
                    want = past.attend(layer, r, turned_q[0], len(past.k[layer][r]))
                    check_close(outs[layer, r].double().cpu().numpy(), want, W.BF16, f"row {r} layer {layer}")

    replay(18)                                                # past the ends of pages
    assert lens.tolist() == [88, 55, 0, 88, 88, 0]

    # row 0 is done; a fork of row 3 takes an empty row; the pool is compacted in two bounded steps, and the same graph goes on
    B.mc_kv_pages_free(counts, tables, PAGE, lens, ints([0]), report)
    B.mc_kv_pages_fork(counts, tables, PAGE, lens, ints([3]), ints([5]), moves[:1], report, pages_ws)
    B.mc_kv_copy_pages(k_pools, v_pools, pages, HKV * PAGE * D * 2, moves[:1], report)
    past.free(0)
    past.fork(3, 5)
    add.copy_(ints([0, 1, 0, 1, 1, 1]))
    for most in (3, pages):
        listed = ints([[0, 0]] * most)
        B.mc_kv_pages_compact(counts, listed, report, pages_ws)
        B.mc_kv_copy_pages(k_pools, v_pools, pages, HKV * PAGE * D * 2, listed, report)
        B.mc_kv_pages_remap(counts, tables, PAGE, lens, listed, report)
    live = int((counts > 0).sum())
    assert bool((counts[:live] > 0).all()) and report.tolist()[0] > 0
    replay(12)
    used = {int(x) for r, n in enumerate(lens.tolist()) for x in tables[r, : -(-n // PAGE)].tolist()}
    assert int((counts > 0).sum()) == others + len(used)

    B.mc_kv_pages_free(counts, tables, PAGE, lens, ints([1, 3, 4, 5]), report)
    assert report.tolist() == [len(used), 0, 0, 0] and int((counts > 0).sum()) == others
