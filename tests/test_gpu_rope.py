"""Head norms, rotation and append in one pass, against the formulas in 64 bits; the pools slot by slot."""
import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from rope_util import assert_rounded, turned

pytestmark = pytest.mark.gpu
DEV, PAGE = "cuda:0", 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Call:
    """Inputs of a batch on the GPU, the pools filled with a pattern, and what the pass has to leave."""

    def __init__(self, dtype, heads, dim, prefix, new, rotary, pairs, norm, scaling=B.MC_ROPE_PLAIN, gain=1.0, fused=True, seed=0, eps=1e-6):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.t, (self.Hq, self.Hkv), self.D = TYPES[dtype], heads, dim
        self.prefix, self.new, self.T = prefix, new, sum(new)
        self.wide = max(1, max(-(-(p + c) // PAGE) for p, c in zip(prefix, new)))
        # only pages that are written are a request's own; the others' entries must not matter to a write
        written = [(p // PAGE, -(-(p + c) // PAGE)) for p, c in zip(prefix, new)]
        self.pages = 3 + sum(hi - lo for (lo, hi), c in zip(written, new) if c)
        ids = list(3 + torch.randperm(self.pages - 3, generator=torch.Generator().manual_seed(seed)).numpy())
        table = np.zeros((len(new), self.wide), np.int32)
        for r, (lo, hi) in enumerate(written):
            for j in range(lo, hi if new[r] else lo):
                table[r, j] = ids.pop()
        self.table_host = table
        self.table = torch.from_numpy(table).to(DEV)
        wide = (self.Hq + 2 * self.Hkv) * dim
        rows = torch.randn((max(self.T, 1), wide), device=DEV, generator=gen, dtype=self.t)[: self.T]
        self.q, self.k, self.v = rows.split((self.Hq * dim, self.Hkv * dim, self.Hkv * dim), dim=1)
        if not fused:
            self.q, self.k, self.v = (x.reshape(self.T, -1, dim).contiguous() for x in (self.q, self.k, self.v))
        self.qw, self.kw = (((1 + 0.3 * torch.randn(dim, device=DEV, generator=gen)).to(self.t) if norm else None) for _ in range(2))
        self.p = B.attn_params(self.Hq, self.Hkv, dim, PAGE, self.pages, dtype)
        self.rope = B.rope_params(rotary, B.MC_ROPE_PAIRS if pairs else B.MC_ROPE_HALF, scaling=scaling, factor=4.0, gain=gain, norm_eps=eps)
        self.rotary, self.pairs, self.gain, self.eps = rotary, pairs, gain, eps
        self.k_pool, self.v_pool = (torch.full((self.pages, self.Hkv, PAGE, dim), x, dtype=self.t, device=DEV) for x in (-7.0, 9.0))
        self.q_out = torch.full((self.T, self.Hq, dim), 5.0, dtype=self.t, device=DEV)
        self.row_of = np.repeat(np.arange(len(new)), new)
        self.pos = np.concatenate([np.arange(p, p + c) for p, c in zip(prefix, new)]) if self.T else np.zeros(0, np.int64)

    def args(self):
        return (self.q, self.k, self.v, self.qw, self.kw, self.q_out, self.k_pool, self.v_pool, self.table)

    def paged(self, stream=None):
        ws = torch.empty(B.mc_kv_append_workspace_bytes(len(self.new)), dtype=torch.uint8, device=DEV)
        B.mc_kv_rope_append_paged(self.p, self.rope, *self.args(), self.prefix, self.new, ws, stream)
        return ws

    def check(self, tokens=None, what=""):
        """All tokens, or those listed, have been written and nothing else has."""
        torch.cuda.synchronize()
        tokens = np.arange(self.T) if tokens is None else np.asarray(tokens, np.int64)
        inv = list(self.rope.inv_freq)
        rest = dict(pos=self.pos[tokens], inv_freq=inv, rotary=self.rotary, pairs=self.pairs, gain=self.gain, eps=self.eps)
        w = [None if x is None else x.double().cpu().numpy() for x in (self.qw, self.kw)]
        q, k = (x.double().cpu().numpy().reshape(self.T, -1, self.D)[tokens] for x in (self.q, self.k))
        assert_rounded(self.q_out[torch.from_numpy(tokens).to(DEV)], *turned(q, w[0], **rest), self.t, what + " q")
        page = torch.from_numpy(self.table_host[self.row_of[tokens], self.pos[tokens] // PAGE].astype(np.int64)).to(DEV)
        slot = torch.from_numpy(self.pos[tokens] % PAGE).to(DEV)
        assert_rounded(self.k_pool[page, :, slot], *turned(k, w[1], **rest), self.t, what + " k")
        index = torch.from_numpy(tokens).to(DEV)
        assert torch.equal(self.v_pool[page, :, slot], self.v.reshape(self.T, self.Hkv, self.D)[index])
        # the other slots and rows hold the pattern
        for pool, mark in ((self.k_pool, -7.0), (self.v_pool, 9.0)):
            rest_of = pool.clone()
            rest_of[page, :, slot] = mark
            assert bool((rest_of == mark).all())
        others = np.setdiff1d(np.arange(self.T), tokens)
        assert bool((self.q_out[torch.from_numpy(others).to(DEV)] == 5.0).all())


SHAPES = [("bf16", (8, 1), 128), ("bf16", (64, 8), 128), ("bf16", (5, 5), 64), ("bf16", (12, 4), 64), ("f32", (4, 1), 64), ("f32", (1, 1), 64)]


@pytest.mark.parametrize("dtype,heads,dim", SHAPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rotary", [0, 16, 48, "all"])
def test_layouts_and_parts_of_a_head(dtype, heads, dim, pairs, rotary):
    rotary = dim if rotary == "all" else rotary
    for norm, prefix, new in ((True, [0, 37, 16], [3, 1, 17]), (False, [1000], [5])):
        c = Call(dtype, heads, dim, prefix, new, rotary, pairs, norm, gain=1.25 if norm else 1.0, fused=norm, seed=rotary)
        c.paged()
        c.check()


@pytest.mark.parametrize("dtype,heads,dim", SHAPES)
@pytest.mark.parametrize("prefix,new", [([0], [1]), ([15], [2]), ([0, 5, 0, 31], [0, 0, 700, 0]), ([7, 0, 100, 3], [33, 64, 0, 1]),
                                        ([4096], [1111])])
def test_lengths(dtype, heads, dim, prefix, new):
    c = Call(dtype, heads, dim, prefix, new, 32, False, True, fused=len(new) == 1, seed=len(new))
    c.paged()
    c.check()


@pytest.mark.parametrize("n", [64, 65, 200])
def test_many_requests(n):
    """Up to 64 travel with the launch, more are uploaded; requests without new tokens among them."""
    new = [(r * 7) % 5 for r in range(n)]
    c = Call("bf16", (16, 2), 128, [r * 13 % 90 for r in range(n)], new, 128, True, True, seed=n)
    c.paged()
    c.check()


def test_no_tokens():
    c = Call("bf16", (8, 1), 128, [5, 9], [0, 0], 128, False, True)
    c.paged()
    torch.cuda.synchronize()
    assert bool((c.k_pool == -7.0).all()) and bool((c.v_pool == 9.0).all())


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("scaling", [B.MC_ROPE_PLAIN, B.MC_ROPE_LINEAR, B.MC_ROPE_BASE, B.MC_ROPE_BY_PARTS])
def test_far_positions(dtype, dim, scaling):
    """A million tokens in, where an angle in 32 bits is off by a twentieth of a radian."""
    c = Call(dtype, (4, 2), dim, [1048573, 130000], [40, 9], dim, False, False, scaling=scaling, seed=3)
    c.paged()
    c.check()


def test_rows_of_zeros_and_large_values():
    c = Call("f32", (2, 1), 64, [3], [6], 64, True, True, eps=1e-6, fused=False)
    c.q[1] = 0.0
    c.k[2] *= 1e12
    c.paged()
    c.check()


@pytest.mark.parametrize("kv_splits", [0, 2])
def test_prepared(kv_splits):
    one, two = (Call("bf16", (16, 2), 128, [200, 0, 33], [100, 45, 0], 64, False, True, seed=8) for _ in range(2))
    one.paged()
    ws = torch.empty(B.mc_prefill_attn_split_workspace_bytes(two.p, 3, 145, 2), dtype=torch.uint8, device=DEV)
    plan = B.mc_prefill_attn_prepare(two.p, two.prefix, two.new, kv_splits, ws)
    B.mc_kv_rope_append_run(two.p, plan, two.rope, *two.args(), ws)
    torch.cuda.synchronize()
    for a, b in ((one.q_out, two.q_out), (one.k_pool, two.k_pool), (one.v_pool, two.v_pool)):
        assert torch.equal(a, b)
    two.check()


@pytest.mark.parametrize("dtype,heads,dim", SHAPES)
@pytest.mark.parametrize("n", [1, 3, 77])
def test_one_token_a_row(dtype, heads, dim, n):
    """Lengths on the device; padding rows and lengths past the table leave everything as it was."""
    pos = [(r * 37) % 250 for r in range(n)]
    c = Call(dtype, heads, dim, pos, [1] * n, 32, False, True, seed=n, fused=n != 3)
    lens = [p + 1 for p in pos]
    out = [r for r in range(n) if r % 5 == 3]
    for i, r in enumerate(out):
        lens[r] = (0, -4, c.wide * PAGE + 1, 2 ** 31 - 1)[i % 4]
    d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    B.mc_kv_rope_append_decode(c.p, c.rope, *c.args(), d)
    c.check([r for r in range(n) if r not in out])


def test_one_token_is_what_a_chunk_of_one_is():
    pos = [5, 130, 77]
    one, two = (Call("bf16", (16, 4), 64, pos, [1, 1, 1], 48, True, True, seed=1) for _ in range(2))
    one.paged()
    B.mc_kv_rope_append_decode(two.p, two.rope, *two.args(), torch.tensor([p + 1 for p in pos], dtype=torch.int32, device=DEV))
    for a, b in ((one.q_out, two.q_out), (one.k_pool, two.k_pool), (one.v_pool, two.v_pool)):
        assert torch.equal(a, b)


def test_in_place_and_on_another_stream():
    a = Call("bf16", (16, 2), 128, [9], [300], 128, False, True, fused=False, seed=4)
    b = Call("bf16", (16, 2), 128, [9], [300], 128, False, True, fused=False, seed=4)
    a.paged()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.q_out = b.q
    keep = b.paged(side)
    side.synchronize()
    assert torch.equal(a.q_out, b.q) and torch.equal(a.k_pool, b.k_pool)
    del keep


def test_replayed_while_lengths_grow():
    n, steps = 4, 5
    pos = [14, 0, 40, 31]
    c = Call("bf16", (8, 2), 128, pos, [steps] * n, 128, False, True, seed=6)
    rows = [x.reshape(n, steps, -1, 128) for x in (c.q, c.k, c.v)]
    now = [torch.zeros_like(x[:, 0]).contiguous() for x in rows]
    lens = torch.tensor([p for p in pos], dtype=torch.int32, device=DEV)
    q_out = torch.zeros((n, 8, 128), dtype=c.t, device=DEV)

    def step():
        lens.add_(1)
        B.mc_kv_rope_append_decode(c.p, c.rope, *now, c.qw, c.kw, q_out, c.k_pool, c.v_pool, c.table, lens)

    step()                                                    # (the library is loaded outside the capture)
    lens.copy_(torch.tensor(pos, dtype=torch.int32))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        for to, x in zip(now, rows):
            to.copy_(x[:, i])
        graph.replay()
        c.q_out.view(n, steps, 8, 128)[:, i] = q_out
        torch.cuda.synchronize()
    c.check()
