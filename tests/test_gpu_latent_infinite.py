"""A key whose score is NaN or +inf makes NaN of the rows that see it, in both forms of attention over a cache of latent vectors, and of no others."""
import pytest
import torch

from latent_util import P, PAGE, absorbed_reference, assert_near, gen, params, prefill_reference, randn, tables
from paper_2407_00079_amd import binding as B
from test_gpu_latent_decode import attend as absorbed
from test_gpu_latent_prefill import attend as expanded
from test_gpu_latent_prefill import inputs

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def hit(out, lse, rows):
    return bool(torch.isnan(out[rows].float()).all()) and bool(torch.isnan(lse[rows]).all())


# prefix, new tokens, the key: in whole tiles, in the loop over tiles that all rows see, near the diagonal, and in row tiles that are cut along the keys
@pytest.mark.parametrize("prefix,new,bad", [(70, 150, 160), (70, 150, 3), (1000, 300, 130), (1000, 300, 1100), (0, 600, 300), (2500, 40, 40), (2500, 40, 1300),
                                            (2500, 40, 2510)])
@pytest.mark.parametrize("what", ["k", "r"])
@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("head_dim", [128, 64])
def test_expanded(prefix, new, bad, what, value, head_dim):
    heads, R = 2, 256
    p, q, k, v, pool, table = inputs(prefix + bad, heads, R, head_dim, [prefix], [new])
    column = 5 if what == "k" else head_dim + 9
    q[:, :, column] = q[:, :, column].abs() + 0.5              # (times +inf: +inf)
    want, want_lse, out_off, lse_off = prefill_reference(q, k, v, pool, table, [prefix], [new], R, (head_dim + P) ** -0.5)
    if what == "k":
        k[bad, :, column] = value
    else:
        pool[table[0, bad // PAGE].long(), bad % PAGE, R + 9] = value
    out, lse = expanded(p, q, k, v, pool, table, [prefix], [new])
    before = max(0, bad - prefix)                              # rows that do not see it
    assert_near(lse[:before], want_lse[:before], lse_off[:before], "lse of rows before it")
    assert_near(out[:before], want[:before], out_off[:before], "out of rows before it")
    assert hit(out, lse, slice(before, new))


# which column: of c, which is a value, too, or of r; how far before a row's end the key stands
@pytest.mark.parametrize("heads,tokens", [(16, 1), (10, 3), (16, 4), (40, 2)])
@pytest.mark.parametrize("column", [7, 512 + 9])
@pytest.mark.parametrize("back", [1, 2, 3, 64, 70])
@pytest.mark.parametrize("value", [NAN, INF])
def test_absorbed(heads, tokens, column, back, value):
    R = 512
    lens = [130, 75, 200, 5000, 71]
    g = gen(heads + back)
    table, pages = tables(g, lens)
    pool, q = randn(g, pages, PAGE, R + P), randn(g, len(lens) * tokens, heads, R + P)
    q[:, :, column] = q[:, :, column].abs() + 0.5
    want, want_lse, out_off, lse_off = absorbed_reference(q, pool, table, lens, tokens, R, (128 + P) ** -0.5)
    for r, n in enumerate(lens):
        at = n - back
        pool[table[r, at // PAGE].long(), at % PAGE, column] = value
    out, lse = absorbed(params(heads, R, 128, pages), q, pool, table, lens, tokens)
    for r in range(len(lens)):
        blind = max(0, tokens - back)                          # tokens that do not see it
        none, some = slice(r * tokens, r * tokens + blind), slice(r * tokens + blind, (r + 1) * tokens)
        assert_near(lse[none], want_lse[none], lse_off[none], "lse of tokens before it")
        assert_near(out[none], want[none], out_off[none], "out of tokens before it")
        assert hit(out, lse, some)


def test_one_row_of_many_stretches():
    """A key of one long row's early part, whose parts are joined by a launch of their own."""
    g, R, heads, n = gen(5), 512, 16, 40000
    table, pages = tables(g, [n])
    pool, q = randn(g, pages, PAGE, R + P), randn(g, 1, heads, R + P)
    q[:, ::2, 3], q[:, 1::2, 3] = q[:, ::2, 3].abs() + 0.5, 0.0
    p = params(heads, R, 128, pages)
    pool[table[0, 700].long(), 2, 3] = INF                     # every second head's score +inf, the others' NaN (0 times it)
    out, lse = absorbed(p, q, pool, table, [n], 1)
    assert hit(out, lse, slice(0, 1))
