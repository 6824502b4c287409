"""Attention of one new token a row, lengths on the device, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from decode_util import PAGE, assert_near, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Call:
    def __init__(self, dtype, heads, dim, lens, seed=0, wide=None, sharp=1.0, nan=True):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.t, (self.Hq, self.Hkv), self.D, self.lens = TYPES[dtype], heads, dim, list(lens)
        real = [max(0, n) for n in lens]
        need = [-(-n // PAGE) for n in real]
        self.wide = wide or max(1, max(need))
        self.pages = sum(need) + 3
        ids = (torch.randperm(self.pages, device=DEV, generator=gen)).to(torch.int32)
        # entries past a row's pages must not be looked at: far outside the pool
        self.table = torch.full((len(lens), self.wide), 2 ** 30, dtype=torch.int32, device=DEV)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = ids[at: at + n]
            at += n
        shape = (self.pages, self.Hkv, PAGE, dim)
        self.q = torch.randn((len(lens), self.Hq, dim), device=DEV, generator=gen, dtype=self.t) * sharp
        self.k, self.v = (torch.randn(shape, device=DEV, generator=gen, dtype=self.t) for _ in range(2))
        if nan:                                               # slots past a length, and pages of no row
            for r, n in enumerate(real):
                if n % PAGE:
                    self.k[self.table[r, n // PAGE].long(), :, n % PAGE:] = math.nan
                    self.v[self.table[r, n // PAGE].long(), :, n % PAGE:] = math.nan
            self.k[ids[at:].long()] = math.nan
            self.v[ids[at:].long()] = math.inf
        self.p = B.attn_params(self.Hq, self.Hkv, dim, PAGE, self.pages, dtype)
        self.d_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.out = torch.full((len(lens), self.Hq, dim), math.nan, dtype=self.t, device=DEV)
        self.lse = torch.full((len(lens), self.Hq), math.nan, device=DEV)
        self.ws = torch.full((B.mc_decode_attn_workspace_bytes(self.p, len(lens)),), 255, dtype=torch.uint8, device=DEV)

    def run(self, lse=True, stream=None):
        B.mc_decode_attn_paged(self.p, self.q, self.k, self.v, self.table, self.d_lens, self.out, self.lse if lse else None, self.ws, stream)

    def check(self, lens=None, what=""):
        scale = self.p.softmax_scale or 1 / math.sqrt(self.D)
        out, lse, out_off, lse_off = reference(self.q, self.k, self.v, self.table, self.lens if lens is None else lens, scale)
        assert_near(self.out, out, out_off, what + " out")
        assert_near(self.lse, lse, lse_off, what + " lse")


KINDS = [("bf16", 128), ("bf16", 64), ("f32", 64)]


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("heads", [(1, 1), (8, 1), (6, 3), (40, 8), (16, 1), (17, 1), (66, 2)])
@pytest.mark.parametrize("lens", [[1], [0], [15, 16, 17], [31, 32, 33, 0, 1], [0, 0, 500, 0], [3000], [64] * 40])
def test_heads_and_lengths(dtype, dim, heads, lens):
    c = Call(dtype, heads, dim, lens, seed=len(lens) + heads[0])
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("seed", range(6))
def test_uneven_batches(dtype, dim, seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 90))
    lens = [int(x) if rng.random() > 0.1 else 0 for x in np.exp(rng.uniform(0, math.log(4000), n))]
    heads = [(8, 1), (12, 4), (64, 8), (5, 5), (32, 2), (14, 2)][seed]
    c = Call(dtype, heads, dim, lens, seed=seed, wide=max(1, -(-max(lens) // PAGE)) + seed)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("heads,lens", [((8, 1), [70001]), ((64, 8), [40000, 3]), ((2, 2), [30000, 0, 16384, 1])])
def test_long(dtype, dim, heads, lens):
    c = Call(dtype, heads, dim, lens, seed=9)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("n", [511, 512, 513, 3000, 20000])
def test_many_rows(dtype, dim, n):
    c = Call(dtype, (2, 1), dim, [(r * 11) % 70 for r in range(n)], seed=n)
    c.run()
    c.check()


@pytest.mark.parametrize("blocks", [2047, 2048, 2049, 4095, 4097])
def test_around_the_number_of_waves(blocks):
    """One row whose blocks are about as many as the waves that share them out, and rows of one block each."""
    c = Call("bf16", (4, 1), 128, [blocks * 32 - 5], seed=blocks)
    c.run()
    c.check()
    c = Call("bf16", (4, 1), 64, [7] * blocks, seed=blocks)
    c.run()
    c.check()


def test_lengths_without_room_in_the_table():
    lens = [40, 33, -7, 48, 2 ** 31 - 1, 49, 1]
    c = Call("bf16", (8, 2), 128, [min(n, 48) for n in lens], seed=2, wide=3)
    c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    c.run()
    c.check([n if n <= 48 else 0 for n in lens])
    none = Call("bf16", (8, 2), 128, [0, 0], seed=2)
    none.table = none.table[:, :0].contiguous()
    with pytest.raises(B.McError):                            # a table without columns has no address
        none.run()


@pytest.mark.parametrize("dtype,dim", KINDS)
def test_sharp_scores_and_a_scale_of_its_own(dtype, dim):
    c = Call(dtype, (16, 2), dim, [900, 5000, 77], seed=5, sharp=40.0)
    c.run()
    c.check()
    c.p.softmax_scale = 0.37
    c.q /= 40
    c.run()
    c.check()


def test_a_score_that_grows_along_the_keys():
    """The reference of the softmax is raised again and again, in stretches and between them."""
    c = Call("bf16", (8, 1), 128, [20000], seed=3, nan=False)
    ramp = torch.linspace(0.0, 30.0, 20000, device=DEV)
    page, slot = c.table[0].long()[torch.arange(20000, device=DEV) // PAGE], torch.arange(20000, device=DEV) % PAGE
    c.k[page, 0, slot] = (ramp[:, None] / 11.3).to(torch.bfloat16)
    c.q.fill_(1.0)
    c.run()
    c.check()


def test_what_is_not_finite():
    """NaN in a query or a visible key makes its rows NaN and no others; -inf as every score of a row is NaN, as 0 / 0 is."""
    c = Call("bf16", (8, 2), 128, [700, 700, 60, 5000], seed=4)
    c.q[0, 2, 5] = math.nan
    c.k[c.table[1, 30].long(), 1, 4, 9] = math.nan
    c.q[2, 4:].fill_(1.0)
    page = c.table[2, torch.arange(60, device=DEV) // PAGE].long()
    c.k[page, 1, torch.arange(60, device=DEV) % PAGE] = -math.inf
    c.run()
    want = torch.zeros((4, 8), dtype=torch.bool, device=DEV)
    want[0, 2] = want[1, 4:] = want[2, 4:] = True
    assert torch.equal(torch.isnan(c.out).all(-1), want) and torch.equal(torch.isnan(c.out).any(-1), want)
    clean = Call("bf16", (8, 2), 128, [700, 700, 60, 5000], seed=4)
    clean.run()
    assert torch.equal(clean.out[~want], c.out[~want])


def test_same_bits_again_without_lse_and_on_another_stream():
    c = Call("bf16", (64, 8), 128, [5000, 1, 0, 333] * 5, seed=6)
    c.run()
    first = c.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.ws.fill_(7)
    torch.cuda.synchronize()
    c.out.fill_(math.nan)
    side.wait_stream(torch.cuda.current_stream())
    c.run(lse=False, stream=side)
    side.synchronize()
    assert torch.equal(first, c.out)
    c.check()


def test_rows_that_share_pages():
    c = Call("bf16", (8, 1), 128, [1000, 1000, 1000], seed=7)
    c.table[1] = c.table[0]
    c.table[2, :30] = c.table[0, :30]
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("heads,rows,length", [((8, 1), 3, 9000), ((12, 2), 150, 700), ((40, 1), 70, 350)])
def test_shared_pages_give_the_bits_of_copies(dtype, dim, heads, rows, length):
    """Rows on the same full pages, last pages of their own, some rows empty, against the same rows with a copy of every page."""
    lens = [0 if r % 7 == 3 else length - r % 5 for r in range(rows)]
    c = Call(dtype, heads, dim, lens, seed=rows, nan=False)
    full = min(n for n in lens if n) // PAGE
    whole = c.table[0, :full].long()
    for r, n in enumerate(lens):
        if n:
            c.k[c.table[r, :full].long()], c.v[c.table[r, :full].long()] = c.k[whole], c.v[whole]
    c.run()
    apart = c.out.clone(), c.lse.clone()
    for r, n in enumerate(lens):
        if n:
            c.table[r, :full] = c.table[0, :full]
    c.out.fill_(math.nan)
    c.run()
    assert torch.equal(apart[0], c.out) and torch.equal(apart[1], c.lse)
    c.check()


def test_pages_past_32_bits_of_bytes():
    """A pool of 4.6 GB whose last pages are used."""
    c = Call("bf16", (8, 8), 128, [1000, 35], seed=8, nan=False)
    far, near = 140000, c.pages
    k, v = (torch.empty((far, 8, PAGE, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[far - near:], v[far - near:] = c.k, c.v
    c.table = torch.where(c.table < 2 ** 30, c.table + (far - near), c.table)
    c.k, c.v, c.p.num_pages = k, v, far
    c.run()
    c.check()


def test_a_row_of_the_longest_length():
    """2^31 - 1 keys: a table of 2^27 entries that name one page, the last another, whose one slot past the length is not a number.

    Scores are 0, so sums of p and of p V are whole numbers below 2^24 up to a workgroup's (2^23 keys, values up to 7 in the waves'
    2^20); 256 workgroups' parts are joined with at most 40 roundings.  The mean of the values is 3.5, of 2^31 - 1 of them 2^-29 beside."""
    pages, n = 2 ** 27, 2 ** 31 - 1
    p = B.attn_params(1, 1, 64, PAGE, 2, "bf16")
    value = ((torch.arange(PAGE)[:, None] + torch.arange(64)[None, :]) % 8).to(torch.bfloat16)
    k, v = torch.zeros((2, 1, PAGE, 64), dtype=torch.bfloat16), value.expand(2, 1, PAGE, 64).contiguous()
    k[1, 0, 15], v[1, 0, 15] = math.nan, math.nan
    table = torch.zeros((1, pages), dtype=torch.int32, device=DEV)
    table[0, -1] = 1
    out, lse = torch.empty((1, 1, 64), dtype=torch.bfloat16, device=DEV), torch.empty((1, 1), device=DEV)
    ws = torch.empty(B.mc_decode_attn_workspace_bytes(p, 1), dtype=torch.uint8, device=DEV)
    B.mc_decode_attn_paged(p, torch.ones((1, 1, 64), dtype=torch.bfloat16, device=DEV), k.to(DEV), v.to(DEV), table,
                           torch.tensor([n], dtype=torch.int32, device=DEV), out, lse, ws)
    assert bool((out == 3.5).all())
    assert abs(float(lse) - math.log(n)) <= 40 * 2.0 ** -24 + 2.0 ** -22 * (1 + math.log(n))


@pytest.mark.parametrize("dtype,dim", KINDS)
def test_replayed_while_lengths_grow(dtype, dim):
    """A captured call reads the lengths of its replay; rows come and go."""
    c = Call(dtype, (8, 2), dim, [2100, 64, 33, 700], seed=10, nan=False)
    c.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for lens in ([1, 64, 33, 0], [2100, 1, 0, 700], [0, 0, 0, 0], [2000, 63, 32, 699], [2001, 64, 33, 700]):
        c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.out.fill_(math.nan)
        graph.replay()
        replayed = c.out.clone(), c.lse.clone()
        c.check(lens)
        c.run()
        assert torch.equal(replayed[0], c.out) and torch.equal(replayed[1], c.lse)


@pytest.mark.parametrize("dtype,dim", KINDS)
def test_beside_the_prefill_call(dtype, dim):
    """One new token by the prefill's attention with the lengths on the host: the same attention to both kernels' tolerance."""
    lens = [301, 17, 4096]
    c = Call(dtype, (8, 2), dim, lens, seed=11)
    c.run()
    out, lse = torch.zeros_like(c.out), torch.zeros_like(c.lse)
    prefix, new = [n - 1 for n in lens], [1, 1, 1]
    ws = torch.empty(B.mc_prefill_attn_auto_workspace_bytes(c.p, prefix, new), dtype=torch.uint8, device=DEV)
    B.mc_prefill_attn_auto(c.p, c.q, c.k, c.v, c.table, prefix, new, out, lse, ws)
    most = 2e-2 if dtype == "bf16" else 1e-4                  # of tests/gpu_util.py
    assert float((out.float() - c.out.float()).abs().max()) <= most and float((lse - c.lse).abs().max()) <= (4e-3 if dtype == "bf16" else 1e-4)
