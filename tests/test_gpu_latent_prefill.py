"""Expansion and expanded prefill attention of a cache of latent vectors against their definitions in 64 bits."""
import pytest
import torch

from latent_util import (BF16, DEV, F32, HALF, P, PAGE, assert_near, attended, gen, params, prefill_reference, randn, rows_of, tables, workspace)
from paper_2407_00079_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("latent,head_dim,heads,lens", [
    *((*x, lens) for x in ((512, 128, 16), (256, 64, 10), (512, 64, 1), (256, 128, 3), (512, 128, 2)) for lens in ([1], [256], [257], [15, 0, 33, 500, 1], [1] * 100, [0, 7] * 40)),
    (512, 128, 64, [700, 0, 33, 1, 290]), (256, 64, 130, [513, 2, 254]), (256, 128, 64, [3] * 341), (512, 64, 1, [50000, 1, 3]),
    (512, 128, 128, [513, 2, 254, 0, 30]), (256, 128, 512, [300, 0, 299]), (512, 64, 256, [1] * 770)])
def test_expand(latent, head_dim, heads, lens):
    g = gen(heads + len(lens))
    table, pages = tables(g, lens)
    pool = randn(g, pages, PAGE, latent + P)
    weight = randn(g, heads * 2 * head_dim, latent)
    kv = torch.full((sum(lens) + 1, heads, 2 * head_dim), 7.0, dtype=BF16, device=DEV)
    B.mc_latent_expand_paged(params(heads, latent, head_dim, pages), weight, pool, table, lens, kv[:-1], workspace(B.mc_latent_workspace_bytes(len(lens))))
    rows = torch.cat([rows_of(pool, table, r, n)[:, :latent] for r, n in enumerate(lens)])
    w = weight.double().T.contiguous()
    want, size = rows @ w, rows.abs() @ w.abs()
    # fp32 sums of R exact products: R + 2 roundings of values up to Sum |c w|; one rounding to bf16
    assert_near(kv[:-1].flatten(1), want, HALF * want.abs() + (1 + HALF) * (latent + 2) * F32 * size, "kv")
    assert bool((kv[-1] == 7).all())


def attend(p, q, k, v, pool, table, prefix, new, want_lse=True):
    out = torch.full((q.shape[0], p.num_heads, p.head_dim), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((q.shape[0], p.num_heads), 7.0, device=DEV) if want_lse else None
    ws = workspace(B.mc_latent_prefill_attn_workspace_bytes(p, prefix, new))
    B.mc_latent_prefill_attn_paged(p, q, k, v, pool, table, prefix, new, out, lse, ws)
    return out, lse


def inputs(seed, heads, latent, head_dim, prefix, new):
    g = gen(seed)
    lens = [a + b for a, b in zip(prefix, new)]
    table, pages = tables(g, lens)
    pool = randn(g, pages, PAGE, latent + P)
    pool[:, :, :latent] = float("nan")                         # (the latent part is not looked at)
    for r, n in enumerate(lens):                               # nor are slots past the end
        at = torch.arange(n, -(-n // PAGE) * PAGE, device=DEV)
        pool[table[r, at // PAGE].long(), at % PAGE] = float("nan")
    q = randn(g, sum(new), heads, head_dim + P)
    kv = randn(g, sum(lens), heads, 2 * head_dim)
    return params(heads, latent, head_dim, pages), q, kv[:, :, :head_dim], kv[:, :, head_dim:], pool, table


def check(p, q, k, v, pool, table, prefix, new):
    out, lse = attend(p, q, k, v, pool, table, prefix, new)
    want, want_lse, out_off, lse_off = prefill_reference(q, k, v, pool, table, prefix, new, p.latent_dim, (p.head_dim + P) ** -0.5)
    assert_near(lse, want_lse, lse_off, "lse")
    assert_near(out, want, out_off, "out")
    return out, lse


@pytest.mark.parametrize("latent,head_dim", [(512, 128), (256, 64)])
@pytest.mark.parametrize("prefix,new", [([0], [1]), ([0], [64]), ([0], [65]), ([63], [1]), ([64], [33]), ([100], [257]), ([5, 0, 77, 300], [3, 0, 64, 31]),
                                        ([3000], [5]), ([0], [520]), ([1] * 70, [2] * 70), ([1300, 2], [300, 0])])
def test_lengths(latent, head_dim, prefix, new):
    check(*inputs(len(prefix) + sum(new), 3, latent, head_dim, prefix, new), prefix, new)


def test_strides():
    """Keys and values by head, and without distance between tokens of one head."""
    p, q, k, v, pool, table = inputs(4, 5, 512, 128, [40, 9], [70, 3])
    out, lse = attend(p, q, k, v, pool, table, [40, 9], [70, 3])
    by_head = k.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((v.shape[0], 5, 128 + 24), 9.0, dtype=BF16, device=DEV)
    wide[:, :, 8:136] = v
    again = attend(p, q, by_head, wide[:, :, 8:136], pool, table, [40, 9], [70, 3])
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    shared = k[:, :1].expand(-1, 5, -1)                         # one head's keys for all
    check(p, q, shared, v, pool, table, [40, 9], [70, 3])


@pytest.mark.parametrize("what", ["k", "v", "r"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see(what, value):
    """Keys and values that are not finite reach the rows that see them, and no others."""
    prefix, new = [70], [150]
    p, q, k, v, pool, table = inputs(8, 2, 512, 128, prefix, new)
    want, want_lse, out_off, lse_off = prefill_reference(q, k, v, pool, table, prefix, new, 512, 192 ** -0.5)
    bad = 70 + 90
    if what == "r":
        pool[table[0, bad // PAGE].long(), bad % PAGE, 512:] = value
    else:
        (k if what == "k" else v)[bad, :, 5] = value
    out, lse = attend(p, q, k, v, pool, table, prefix, new)
    assert_near(lse[:90], want_lse[:90], lse_off[:90], "lse of rows before it")
    assert_near(out[:90], want[:90], out_off[:90], "out of rows before it")
    if what == "v":                                            # one column of each row behind it, nothing else
        other = [c for c in range(128) if c != 5]
        assert_near(out[90:][:, :, other], want[90:][:, :, other], out_off[90:][:, :, other], "other columns")
        assert_near(lse, want_lse, lse_off, "lse")
        hit = out[90:, :, 5].float()
        assert bool(torch.isnan(hit).all() if value != value else (hit == value).all())


def test_growing_scores():
    p, q, k, v, pool, table = inputs(9, 2, 512, 128, [1200], [40])
    k *= (0.1 + 20.0 * torch.arange(1240, device=DEV) / 1240)[:, None, None].to(BF16)
    check(p, q, k, v, pool, table, [1200], [40])


@pytest.mark.parametrize("prefix,new", [([0], [130]), ([2500], [40])])
def test_scores_of_minus_infinity(prefix, new):
    """A key whose score is -inf counts for nothing; a row that has no others is 0, whether its tile was cut along the keys or not."""
    p, q, k, v, pool, table = inputs(12, 2, 512, 128, prefix, new)
    n = prefix[0] + new[0]
    q[:, :, 7] = q[:, :, 7].abs() + 0.5
    few = torch.arange(0, n, 3, device=DEV)
    lost = torch.ones(n, dtype=torch.bool, device=DEV)
    k[few, :, 7] = -float("inf")
    lost[few] = False
    out, lse = attend(p, q, k, v, pool, table, prefix, new)
    shared = rows_of(pool, table, 0, n)[:, 512:]
    for i in range(new[0]):
        seen = torch.nonzero(lost[: prefix[0] + i + 1])[:, 0]
        if len(seen) == 0:
            assert bool((out[i] == 0).all()) and bool((lse[i] == -float("inf")).all())
            continue
        keys = torch.cat((k[seen].double().transpose(0, 1), shared[seen].expand(2, -1, -1)), 2)
        want, want_lse, out_off, lse_off = attended(q[i].double(), keys, v[seen].double().transpose(0, 1), 192 ** -0.5)
        assert_near(lse[i], want_lse, lse_off, "lse")
        assert_near(out[i], want, out_off, "out")
    k[:, :, 7] = -float("inf")
    out, lse = attend(p, q, k, v, pool, table, prefix, new)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())


def test_most_heads():
    prefix, new = [40, 0], [3, 20]
    check(*inputs(14, 1024, 256, 64, prefix, new), prefix, new)
