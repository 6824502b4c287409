"""Expanded prefill attention where an entry of the request table has several row tiles of 256 rows: more than 64 of them in a call, or more than 64
requests.  (Fewer are entries of their own; test_latent_host_tiles.py holds the plan to what is said here of each case.)"""
import random

import pytest
import torch

from latent_util import BF16, DEV, P, assert_near, attended, rows_of, workspace
from paper_2407_00079_amd import binding as B
from test_gpu_latent_prefill import inputs

pytestmark = pytest.mark.gpu


def among(n, at, prefix, new):
    """n requests of few tokens, among them one of so many."""
    p, c = [(7 * r) % 90 for r in range(n)], [1 + r % 3 if r % 5 else 0 for r in range(n)]
    p[at], c[at] = prefix, new
    return p, c


# heads, R, head_dim, prefixes and new tokens; whether row tiles are cut along the keys
CASES = {
    "one_request": (1, 512, 128, [100], [16700], True),
    "one_request_small_heads": (1, 256, 64, [0], [16640], True),
    "few_requests": (16, 512, 128, [0, 333, 5000, 64, 0], [4000, 4097, 3900, 1, 4352], False),
    "few_requests_small_heads": (15, 256, 64, [16, 0, 2], [7000, 0, 12001], False),
    "uploaded_cut": (3, 512, 128, *among(70, 41, 40000, 700), True),
    "uploaded_cut_small_heads": (2, 512, 64, *among(66, 0, 20011, 513), True),
    "uploaded": (16, 512, 128, *among(70, 69, 11, 600), False),
    "uploaded_several": (12, 256, 64, [r % 7 * 40 for r in range(80)], [300 if r % 4 == 1 else 5 for r in range(80)], False),
}


def sampled(rng, new):
    """Rows to look at: both sides of every end of a row tile and of a wave's rows in some of them, and others."""
    if new <= 8:
        return list(range(new))
    rows = {0, 1, new - 1}
    for end in range(256, new, 256):
        rows |= {end - 1, end}
    for _ in range(30):
        at = rng.randrange(new)
        rows |= {at, min(new - 1, at | 31)}
    return sorted(rows)


@pytest.mark.parametrize("case", CASES)
def test_row_tiles_of_one_entry(case):
    heads, latent, head_dim, prefix, new, _ = CASES[case]
    p, q, k, v, pool, table = inputs(len(case), heads, latent, head_dim, prefix, new)
    T = sum(new)
    ws = workspace(B.mc_latent_prefill_attn_workspace_bytes(p, prefix, new))
    results = []
    for fill in (255, 0):                                      # (as partial results: NaN, and 0)
        ws.fill_(fill)
        out, lse = torch.full((T + 1, heads, head_dim), 7.0, dtype=BF16, device=DEV), torch.full((T + 1, heads), 7.0, device=DEV)
        B.mc_latent_prefill_attn_paged(p, q, k, v, pool, table, prefix, new, out[:T], lse[:T], ws)
        assert bool((out[T] == 7).all()) and bool((lse[T] == 7).all())
        results.append((out[:T], lse[:T]))
    (out, lse), again = results
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert not bool(torch.isnan(out.float()).any()) and not bool(torch.isnan(lse).any())
    rng, scale = random.Random(case), (head_dim + P) ** -0.5
    t0 = n0 = 0
    for r, (before, c) in enumerate(zip(prefix, new)):
        n = before + c
        if c > 0:
            shared = rows_of(pool, table, r, n)[:, latent:]
            keys = torch.cat((k[n0: n0 + n].double().transpose(0, 1), shared.expand(heads, -1, -1)), 2)
            values = v[n0: n0 + n].double().transpose(0, 1)
            for i in sampled(rng, c):
                want, want_lse, out_off, lse_off = attended(q[t0 + i].double(), keys[:, : before + i + 1], values[:, : before + i + 1], scale)
                assert_near(lse[t0 + i], want_lse, lse_off, f"lse of row {i} of request {r}")
                assert_near(out[t0 + i], want, out_off, f"out of row {i} of request {r}")
        t0, n0 = t0 + c, n0 + n
