"""The operators on a cache of latent vectors written out in 64 bits, and what the kernels' arithmetic may be off by."""
import math

import torch

from paper_2407_00079_amd import binding as B

PAGE, P = 16, 64
BF16 = torch.bfloat16
HALF = 2.0 ** -8             # half a step of bf16, relative
F32 = 2.0 ** -24
DEV = "cuda:0"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, device=DEV, generator=g, dtype=torch.float32).to(BF16)


def tables(g, lens, spare=3, rest="any"):
    """Scattered pages for rows of these lengths: (block table, pages in the pool).  Entries past a row's pages name any page, or one that
    no row has."""
    need = [max(0, -(-n // PAGE)) for n in lens]
    pool, wide = sum(need) + spare, max(1, max(need))
    ids = torch.randperm(pool, device=DEV, generator=g).to(torch.int32)
    t = ids[torch.randint(0, pool, (len(lens), wide), device=DEV, generator=g) if rest == "any" else torch.full((len(lens), wide), pool - 1, device=DEV)]
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = ids[at: at + n]
        at += n
    return t.contiguous(), pool


def rows_of(pool, table, r, n):
    return pool[table[r, : -(-n // PAGE)].long()].flatten(0, 1)[:n].double()


def lens_tensor(lens):
    return torch.tensor(lens, dtype=torch.int32, device=DEV)


def workspace(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


def attended(q, k, v, scale):
    """Queries [H, K] over keys [n, K] or [H, n, K] and values [n, R] or [H, n, R], in 64 bits: out, lse and the bounds on their errors.

    Units of 2^-24: a score's products are exact and summed in fp32, at most K + 2 roundings of values up to Sum |q k|; the exponent is rounded once
    more, exp2 and log2 are within 2: a probability is off by (K + 4) max Sum |q k| scale + 4 relative, its sum over n keys by n / 8 + 16
    additions of what the lanes and waves hold.  A probability is rounded to bf16 before it meets a value (half a step: 2^-8), the sum takes it as it
    was.  The output is the quotient of two such sums, rounded once."""
    H, K = q.shape
    k = k.expand(H, -1, -1) if k.dim() == 2 else k
    v = v.expand(H, -1, -1) if v.dim() == 2 else v
    score = torch.matmul(k, q[:, :, None])[..., 0] * scale
    lse = torch.logsumexp(score, 1)
    p = torch.exp(score - lse[:, None])
    size = torch.matmul(k.abs(), q.abs()[:, :, None])[..., 0].amax(1) * scale
    rel = ((K + 4) * size + 4 + k.shape[1] / 8 + 16) * F32
    out = torch.matmul(p[:, None, :], v)[:, 0]
    spread = torch.matmul(p[:, None, :], v.abs())[:, 0]
    off = (2 * rel[:, None] + HALF) * spread
    return out, lse, HALF * out.abs() + (1 + HALF) * off, rel + 2.0 ** -22 * (1 + lse.abs())


def assert_near(got, want, most, what):
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - most)
    bad = ~(off <= 0)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} values past their bound, the first at {bad.nonzero()[0].tolist()}: " \
                                f"{got[bad][0].item()} against {want[bad][0].item()} +- {most[bad][0].item():.3g}"


def absorbed_reference(q, pool, table, lens, tokens, R, scale):
    """q [rows * tokens, H, R + P]: (out, lse, their bounds)."""
    T, H, _ = q.shape
    out = torch.zeros((T, H, R), dtype=torch.float64, device=DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=DEV)
    out_off, lse_off = torch.zeros_like(out), torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for r, n in enumerate(lens):
        if not 0 < n <= table.shape[1] * PAGE:
            continue
        rows = rows_of(pool, table, r, n)
        for t in range(tokens):
            seen = n - tokens + t + 1
            if seen > 0:
                i = r * tokens + t
                out[i], lse[i], out_off[i], lse_off[i] = attended(q[i].double(), rows[:seen], rows[:seen, :R], scale)
    return out, lse, out_off, lse_off


def prefill_reference(q, k, v, pool, table, prefix, new, R, scale):
    """(out, lse, their bounds) of chunks over expanded keys and values."""
    T, H, _ = q.shape
    D = v.shape[2]
    out = torch.zeros((T, H, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((T, H), dtype=torch.float64, device=DEV)
    out_off, lse_off = torch.zeros_like(out), torch.zeros_like(lse)
    t0 = n0 = 0
    for r, (p, c) in enumerate(zip(prefix, new)):
        n = p + c
        if c > 0:
            shared = rows_of(pool, table, r, n)[:, R:]
            keys = torch.cat((k[n0: n0 + n].double().transpose(0, 1), shared.expand(H, -1, -1)), 2)
            values = v[n0: n0 + n].double().transpose(0, 1)
            for i in range(c):
                at = t0 + i
                out[at], lse[at], out_off[at], lse_off[at] = attended(q[at].double(), keys[:, : p + i + 1], values[:, : p + i + 1], scale)
        t0, n0 = t0 + c, n0 + n
    return out, lse, out_off, lse_off


def params(heads, latent, head_dim, pages, scale=0.0):
    return B.latent_params(heads, latent, P, head_dim, PAGE, pages, "bf16", scale)
