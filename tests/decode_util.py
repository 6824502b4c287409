"""Decode attention written out in 64 bits, and what the kernel's arithmetic may be off by."""
import math

import torch

PAGE = 16
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def reference(q, k_pool, v_pool, table, lens, scale):
    """Per row and head: out, lse, and the bounds on their errors (all in 64 bits, on the inputs' device).

    Units of 2^-24: a score's products are exact and summed in fp32, at most D + 2 roundings of values up to Sum |q k|; the
    exponent that goes into exp2 is rounded once more, relative to the distance from the reference (taken as the largest score in
    magnitude); exp2 and log2 are within 2.  So a probability is off by (D + 4) max Sum |q k| scale + 4 relative, its sum over n
    keys by n / 8 + 16 additions of what the lanes hold.  bf16: p enters as two bf16 values, 2^-16 of it is lost.  The output is
    the quotient of two such sums, rounded once."""
    B, Hq, D = q.shape
    Hkv = k_pool.shape[1]
    G = Hq // Hkv
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=q.device)
    out_off, lse_off = torch.zeros_like(out), torch.zeros((B, Hq), dtype=torch.float64, device=q.device)
    half = HALF_STEP[q.dtype]
    for r, n in enumerate(lens):
        if not 0 < n <= table.shape[1] * PAGE:
            continue
        ids = table[r, : -(-n // PAGE)].long()
        k, v = (p[ids].permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n].double() for p in (k_pool, v_pool))
        x = q[r].double().reshape(Hkv, G, D)
        score = torch.bmm(x, k.transpose(1, 2).contiguous()) * scale
        lse_r = torch.logsumexp(score, 2)
        p = torch.exp(score - lse_r[..., None])
        size = torch.bmm(x.abs(), k.abs().transpose(1, 2).contiguous()).amax(2) * scale              # [Hkv, G]
        rel = ((D + 4) * size + 4 + n / 8 + 16) * 2.0 ** -24
        o = torch.bmm(p, v)
        spread = torch.bmm(p, v.abs())
        out[r], lse[r] = o.reshape(Hq, D), lse_r.reshape(Hq)
        lost = 2.0 ** -16 if q.dtype == torch.bfloat16 else 0.0
        off = 2 * (rel + lost)[..., None] * spread
        out_off[r] = (half * o.abs() + (1 + half) * off).reshape(Hq, D)
        lse_off[r] = (rel + 2.0 ** -22 * (1 + lse_r.abs())).reshape(Hq)
    return out, lse, out_off, lse_off


def assert_near(got, want, most, what):
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - most)
    bad = ~(off <= 0)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} values past their bound, the first at {bad.nonzero()[0].tolist()}: " \
                                f"{got[bad][0].item()} against {want[bad][0].item()} +- {most[bad][0].item():.3g}"
