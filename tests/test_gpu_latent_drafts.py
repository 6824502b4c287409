"""Steps that verify drafted tokens of which some are refused: the page state's lengths say what a row holds, a second tensor which of its tokens count."""
import random

import torch
import pytest

from latent_util import BF16, DEV, P, PAGE, absorbed_reference, assert_near, gen, params, randn, rows_of, workspace
from paper_2407_00079_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS, WIDE, PAGES, TOKENS = 6, 20, 64, 4


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


class State:
    def __init__(self, g, heads, R, head_dim):
        self.g, self.heads, self.R = g, heads, R
        self.p, self.rope = params(heads, R, head_dim, PAGES), B.rope_params(P, B.MC_ROPE_HALF)
        self.scale = (head_dim + P) ** -0.5
        self.pool = torch.full((PAGES, PAGE, R + P), float("nan"), dtype=BF16, device=DEV)
        self.counts, self.held, self.lens, self.table = ints([0] * PAGES), ints([0] * ROWS), ints([0] * ROWS), ints([[0] * WIDE] * ROWS)
        self.active, self.add, self.now, self.report = ints([0] * ROWS), ints([0] * ROWS), ints([0] * ROWS), ints([0] * 4)
        self.pages_ws = workspace(B.mc_kv_pages_workspace_bytes(PAGES, ROWS))
        self.attn_ws = workspace(B.mc_latent_decode_attn_workspace_bytes(self.p, ROWS, TOKENS))
        self.q, self.q_all = torch.zeros((ROWS * TOKENS, heads, P), dtype=BF16, device=DEV), torch.zeros((ROWS * TOKENS, heads, R + P), dtype=BF16, device=DEV)
        self.down = torch.zeros((ROWS * TOKENS, R + P), dtype=BF16, device=DEV)
        self.out, self.lse = torch.zeros((ROWS * TOKENS, heads, R), dtype=BF16, device=DEV), torch.zeros((ROWS * TOKENS, heads), device=DEV)
        self.past = {}                                         # rows of the cache that count

    def prompt(self, lens):
        B.mc_kv_pages_grow(self.counts, self.table, PAGE, self.held, ints(lens), self.report, self.pages_ws)
        assert self.report.tolist()[1] == 0
        T, ws = sum(lens), workspace(B.mc_latent_workspace_bytes(ROWS))
        q, down = randn(self.g, T, self.heads, P), randn(self.g, T, self.R + P)
        B.mc_latent_append_paged(self.p, self.rope, q, down, None, q, self.pool, self.table, [0] * ROWS, lens, ws)
        self.lens.copy_(ints(lens))
        self.active.copy_(ints([n > 0 for n in lens]))
        for r, n in enumerate(lens):
            self.past[r] = rows_of(self.pool, self.table, r, n)

    def step(self):
        """Drafts of all rows, nothing uploaded or waited for: rows hold what they have and TOKENS more."""
        torch.sub(self.lens, self.held, out=self.add)
        self.add.add_(TOKENS).mul_(self.active)
        B.mc_kv_pages_grow(self.counts, self.table, PAGE, self.held, self.add, self.report, self.pages_ws)
        torch.add(self.lens, TOKENS, out=self.now)
        self.now.mul_(self.active).mul_(self.report[1:2] == 0)
        B.mc_latent_append_decode(self.p, self.rope, self.q, self.down, None, self.q_all[:, :, self.R:], self.pool, self.table, self.now, TOKENS)
        B.mc_latent_decode_attn_paged(self.p, self.q_all, self.pool, self.table, self.now, TOKENS, self.out, self.lse, self.attn_ws)

    def verify(self, rng):
        """Looks the step over, then takes 1 to TOKENS of each row's tokens."""
        now, held = self.now.tolist(), self.held.tolist()
        want, want_lse, out_off, lse_off = absorbed_reference(self.q_all, self.pool, self.table, now, TOKENS, self.R, self.scale)
        assert_near(self.lse, want_lse, lse_off, "lse")
        assert_near(self.out, want, out_off, "out")
        taken = [rng.randint(1, TOKENS) if n > 0 else 0 for n in now]
        self.lens.add_(ints(taken))
        for r, n in enumerate(self.lens.tolist()):
            assert (n == 0) == (held[r] == 0) and n <= held[r]
            if now[r] > 0:
                cache = rows_of(self.pool, self.table, r, n)
                assert torch.equal(cache[: len(self.past[r])], self.past[r]) and not bool(torch.isnan(cache).any())
                self.past[r] = cache
        self.whole()

    def whole(self):
        """Every count is how many rows' tables name the page: none was lost on the way."""
        count, table = [0] * PAGES, self.table.tolist()
        for r, n in enumerate(self.held.tolist()):
            for page in table[r][: -(-n // PAGE)]:
                count[page] += 1
        assert count == self.counts.tolist()


@pytest.mark.parametrize("heads,R,head_dim", [(5, 256, 64), (16, 512, 128)])
def test_refused_drafts(heads, R, head_dim):
    g, rng = gen(heads), random.Random(heads)
    s = State(g, heads, R, head_dim)
    s.step()                                                   # (rows are all padding)
    s.prompt([45, 3, 16, 0, 130, 0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()

    def replay(times):
        for _ in range(times):
            for t in (s.q, s.down, s.q_all):
                t.copy_(randn(g, *t.shape))
            graph.replay()
            torch.cuda.synchronize()
            assert s.report.tolist()[1] == 0
            s.verify(rng)

    replay(12)                                                 # (over the ends of pages, and back over some)
    # another answer to row 0's prompt, at a step behind which both lengths end in one page
    for _ in range(40):
        held, lens = int(s.held[0]), int(s.lens[0])
        if held // PAGE == lens // PAGE and held != lens:
            break
        replay(1)
    assert held // PAGE == lens // PAGE and held != lens
    moves = ints([[0, 0]])
    B.mc_kv_pages_fork(s.counts, s.table, PAGE, s.held, ints([0]), ints([5]), moves, s.report, s.pages_ws)
    assert s.report.tolist()[1] == 0
    B.mc_kv_copy_pages([s.pool], [s.pool], PAGES, PAGE * (R + P) * 2, moves, s.report)
    s.lens[5], s.active[5], s.past[5] = s.lens[0], 1, s.past[0]
    s.whole()
    replay(8)
    # a row is done, what is live goes to the front
    B.mc_kv_pages_free(s.counts, s.table, PAGE, s.held, ints([4]), s.report)
    s.lens[4], s.active[4] = 0, 0
    listed = ints([[-1, -1]] * PAGES)
    B.mc_kv_pages_compact(s.counts, listed, s.report, s.pages_ws)
    B.mc_kv_copy_pages([s.pool], [s.pool], PAGES, PAGE * (R + P) * 2, listed, s.report)
    B.mc_kv_pages_remap(s.counts, s.table, PAGE, s.held, listed, s.report)
    live = int((s.counts > 0).sum())
    assert bool((s.counts[:live] > 0).all())
    replay(6)
    B.mc_kv_pages_free(s.counts, s.table, PAGE, s.held, ints(list(range(ROWS))), s.report)
    assert bool((s.counts == 0).all()) and bool((s.held == 0).all())


def test_growth_that_is_refused():
    """Too few pages for the drafts of all rows: nothing is written, and every length stays; with fewer rows the next step goes on."""
    g, rng = gen(3), random.Random(3)
    s = State(g, 5, 256, 64)
    s.prompt([300, 304, 304, 48, 0, 0])                        # 60 pages of 64
    for t in (s.q, s.down, s.q_all):
        t.copy_(randn(g, *t.shape))
    s.active[4], s.active[5] = 1, 1                            # (two rows that begin: with rows 1, 2 and 3 five pages more)
    pool, held, lens = s.pool.clone(), s.held.tolist(), s.lens.tolist()
    s.step()
    assert s.report.tolist()[1] != 0 and s.now.tolist() == [0] * ROWS and s.held.tolist() == held and s.lens.tolist() == lens
    assert torch.equal(pool.view(torch.int16), s.pool.view(torch.int16)) and bool((s.out == 0).all())
    s.active[4] = 0
    B.mc_kv_pages_free(s.counts, s.table, PAGE, s.held, ints([0]), s.report)
    s.lens[0], s.active[0] = 0, 0
    for _ in range(3):
        for t in (s.q, s.down, s.q_all):
            t.copy_(randn(g, *t.shape))
        s.step()
        assert s.report.tolist()[1] == 0
        s.verify(rng)
