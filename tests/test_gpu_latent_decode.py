"""Absorbed attention over a cache of latent vectors against its definition in 64 bits."""
import pytest
import torch

from latent_util import (BF16, DEV, P, PAGE, absorbed_reference, assert_near, attended, gen, lens_tensor, params, randn, rows_of, tables, workspace)
from paper_2407_00079_amd import binding as B

pytestmark = pytest.mark.gpu


def attend(p, q, pool, table, lens, tokens, want_lse=True, ws=None):
    T, H, R = q.shape[0], p.num_heads, p.latent_dim
    out = torch.full((T, H, R), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((T, H), 7.0, device=DEV) if want_lse else None
    ws = workspace(B.mc_latent_decode_attn_workspace_bytes(p, len(lens), tokens)) if ws is None else ws
    B.mc_latent_decode_attn_paged(p, q, pool, table, lens_tensor(lens), tokens, out, lse, ws)
    return out, lse


def check(heads, latent, head_dim, lens, tokens=1, seed=0, scale=0.0):
    g = gen(seed)
    table, pages = tables(g, lens, rest="unused")
    pool = randn(g, pages, PAGE, latent + P)
    used = torch.zeros((pages, PAGE), dtype=torch.bool, device=DEV)
    for r, n in enumerate(lens):
        at = torch.arange(n, device=DEV)
        used[table[r, at // PAGE].long(), at % PAGE] = True
    pool[~used] = float("nan")                                 # what no row may use as a value
    q = randn(g, len(lens) * tokens, heads, latent + P)
    p = params(heads, latent, head_dim, pages, scale)
    out, lse = attend(p, q, pool, table, lens, tokens)
    want, want_lse, out_off, lse_off = absorbed_reference(q, pool, table, lens, tokens, latent, scale or (head_dim + P) ** -0.5)
    assert_near(lse, want_lse, lse_off, "lse")
    assert_near(out, want, out_off, "out")
    return p, q, pool, table, out, lse


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads", [1, 10, 16, 17, 32, 40, 64, 128, 129])
def test_heads(heads, latent):
    check(heads, latent, 128, [1, 15, 16, 17, 63, 64, 65, 300], seed=heads)


@pytest.mark.parametrize("lens", [[1], [64], [65], [1000], [5000, 1, 4999], [0, 3, 0, 0, 130, 0], [0, 0], [20000], [129] * 300, [1] * 70, [64, 65] * 50, [30] * 300, [-5, 20, 10 ** 9, 7]])
@pytest.mark.parametrize("heads", [16, 64])
def test_lengths(heads, lens):
    g = len(lens) + heads
    if max(lens) > 10 ** 6:                                    # lengths that no table has room for are padding rows'
        real = [n if 0 < n < 10 ** 6 else 0 for n in lens]
        gg = gen(g)
        table, pages = tables(gg, real)
        pool, q = randn(gg, pages, PAGE, 512 + P), randn(gg, len(lens), heads, 512 + P)
        p = params(heads, 512, 128, pages)
        out, lse = attend(p, q, pool, table, lens, 1)
        want, want_lse, out_off, lse_off = absorbed_reference(q, pool, table, real, 1, 512, 192 ** -0.5)
        assert_near(lse, want_lse, lse_off, "lse")
        assert_near(out, want, out_off, "out")
    else:
        check(heads, 512, 128, lens, seed=g)


@pytest.mark.parametrize("tokens", [2, 3, 4, 16])
@pytest.mark.parametrize("heads", [5, 16, 128])
def test_new_tokens(heads, tokens):
    """Each token sees the keys up to its own; rows shorter than the tokens have some that see none; tiles' ends between tokens."""
    check(heads, 512, 128, [1, tokens, 63, 64, 65, 64 + tokens - 1, 128 + 1, 700, 0], tokens=tokens, seed=tokens)


def test_scale_and_no_lse():
    p, q, pool, table, out, lse = check(16, 256, 64, [200, 31], scale=0.3, seed=5)
    again, none = attend(p, q, pool, table, [200, 31], 1, want_lse=False)
    assert none is None and torch.equal(out, again)


def test_growing_scores():
    """Scores that outgrow the reference tile after tile, and by more than 2^8 at once."""
    g = gen(11)
    lens = [1500, 700]
    table, pages = tables(g, lens)
    pool, q = randn(g, pages, PAGE, 512 + P) * 0.1, randn(g, 2, 32, 512 + P)
    for r, n in enumerate(lens):
        at = torch.arange(n, device=DEV)
        pool[table[r, at // PAGE].long(), at % PAGE] *= (0.1 + 30.0 * at / n)[:, None].to(BF16)
    p = params(32, 512, 128, pages)
    out, lse = attend(p, q, pool, table, lens, 1)
    want, want_lse, out_off, lse_off = absorbed_reference(q, pool, table, lens, 1, 512, 192 ** -0.5)
    assert_near(lse, want_lse, lse_off, "lse")
    assert_near(out, want, out_off, "out")


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_a_draft_does_not_see(value):
    """A row of the cache that is not finite reaches the tokens that see it, and no others."""
    g = gen(3)
    lens, tokens, heads = [130, 64, 200], 4, 16
    table, pages = tables(g, lens)
    pool, q = randn(g, pages, PAGE, 512 + P), randn(g, len(lens) * tokens, heads, 512 + P)
    want, want_lse, out_off, lse_off = absorbed_reference(q, pool, table, lens, tokens, 512, 192 ** -0.5)
    for r, n in enumerate(lens):
        pool[table[r, (n - 2) // PAGE].long(), (n - 2) % PAGE, :] = value
    out, lse = attend(params(heads, 512, 128, pages), q, pool, table, lens, tokens)
    for r in range(len(lens)):
        sees = slice(r * tokens, r * tokens + 2)
        assert_near(lse[sees], want_lse[sees], lse_off[sees], "lse of tokens before it")
        assert_near(out[sees], want[sees], out_off[sees], "out of tokens before it")
        if value != value:
            assert bool(torch.isnan(out[r * tokens + 2: (r + 1) * tokens].float()).all())


def test_same_bits_whatever_stands_around():
    g = gen(21)
    lens = [3000, 17, 900]
    table, pages = tables(g, lens)
    pool, q = randn(g, pages, PAGE, 512 + P), randn(g, 3, 64, 512 + P)
    p = params(64, 512, 128, pages)
    ws = workspace(B.mc_latent_decode_attn_workspace_bytes(p, 3, 1))
    first = attend(p, q, pool, table, lens, 1, ws=ws)
    for fill in (0, 255, 127):
        ws.fill_(fill)
        again = attend(p, q, pool, table, lens, 1, ws=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("lens", [[1, 70, 3000], [5000]])
def test_scores_of_minus_infinity(lens):
    """A key whose score is -inf counts for nothing; a row that has no others is 0, whether stretches cut it or not."""
    g = gen(15)
    heads = 16
    table, pages = tables(g, lens)
    pool, q = randn(g, pages, PAGE, 512 + P), randn(g, len(lens), heads, 512 + P)
    q[:, :, 515] = q[:, :, 515].abs() + 0.5
    whole = pool.clone()
    for lost in (2, 1):                                        # every second key, every key
        for r, n in enumerate(lens):
            at = torch.arange(0, n, lost, device=DEV)
            pool[table[r, at // PAGE].long(), at % PAGE, 515] = -float("inf")
        out, lse = attend(params(heads, 512, 128, pages), q, pool, table, lens, 1)
        for r, n in enumerate(lens):
            if lost == 1 or n == 1:
                assert bool((out[r] == 0).all()) and bool((lse[r] == -float("inf")).all())
                continue
            rows = rows_of(whole, table, r, n)[1::2]
            want, want_lse, out_off, lse_off = attended(q[r].double(), rows, rows[:, :512], 192 ** -0.5)
            assert_near(lse[r], want_lse, lse_off, "lse")
            assert_near(out[r], want, out_off, "out")


@pytest.mark.parametrize("heads,tokens", [(1024, 1), (1000, 3), (1024, 16)])
def test_most_heads(heads, tokens):
    check(heads, 256, 64, [70, 3, 0], tokens=tokens, seed=heads)


def test_thousands_of_rows():
    """More rows than 64 a lane, of which few have keys: first, last, in between, and many beside each other."""
    lens = [0] * 4300
    for r in (0, 1, 63, 64, 70, 2047, 4299):
        lens[r] = 1 + 17 * (r % 11)
    lens[900: 1200] = [5] * 300
    lens[3000] = 700
    check(16, 256, 64, lens, seed=33)
