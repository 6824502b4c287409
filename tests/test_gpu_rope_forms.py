"""One row a lane group for few rows, two for many: around the line between them, and the same bits from either."""
import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from test_gpu_rope import Call

pytestmark = pytest.mark.gpu


# rows of two lane groups' worth a workgroup: 32 at 16 lanes a row, 64 at 8; the line is at 512 such workgroups
@pytest.mark.parametrize("dtype,heads,dim,tokens", [
    ("bf16", (64, 8), 128, (204, 205)), ("bf16", (5, 1), 128, (2334, 2341)), ("bf16", (13, 1), 64, (2170, 2200)), ("f32", (2, 2), 64, (2725, 2731)),
    ("f32", (29, 1), 64, (527, 600)), ("bf16", (1, 1), 64, (10901, 10923))])
@pytest.mark.parametrize("pairs", [False, True])
def test_around_the_line(dtype, heads, dim, tokens, pairs):
    for n in tokens:
        c = Call(dtype, heads, dim, [11, 3], [n - 5, 5], dim - 16, pairs, True, seed=n)
        c.paged()
        c.check()


@pytest.mark.parametrize("dtype,heads,dim", [("bf16", (64, 8), 128), ("bf16", (7, 7), 64), ("f32", (12, 3), 64)])
def test_the_same_bits(dtype, heads, dim):
    """A long chunk in one call, and token ranges of it in calls of their own."""
    c = Call(dtype, heads, dim, [21], [3500], dim, False, True, seed=4)
    c.paged()
    whole = c.q_out.clone(), c.k_pool.clone(), c.v_pool.clone()
    for x, mark in zip((c.q_out, c.k_pool, c.v_pool), (5.0, -7.0, 9.0)):
        x.fill_(mark)
    ws = torch.empty(B.mc_kv_append_workspace_bytes(1), dtype=torch.uint8, device="cuda:0")
    for lo in range(0, 3500, 100):
        part = slice(lo, lo + 100)
        B.mc_kv_rope_append_paged(c.p, c.rope, c.q[part], c.k[part], c.v[part], c.qw, c.kw, c.q_out[part], c.k_pool, c.v_pool, c.table, [21 + lo], [100], ws)
    assert all(torch.equal(a, b) for a, b in zip(whole, (c.q_out, c.k_pool, c.v_pool)))
    c.check(np.arange(3500))
