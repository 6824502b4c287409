"""What a serving program does with a cache of latent vectors, as cases that can be timed.

A token leaves one vector in the cache: ``latent`` numbers that the keys and values of all heads are made from, and ``ROPE`` numbers, rotated
by its position, that all heads' keys share.  A case is a dict of plain values.  Four kinds:

  append   projections become cache entries: the latent part is normalised, the shared key part and every head's query part are rotated,
           [latent, key] goes into its page slot.  ``form`` is "prompt" (a chunk a request) or "tokens" (``tokens`` new ones a row, lengths on
           the device)
  absorb   ``tokens`` new tokens a row attend to the row's latent vectors themselves, lengths on the device
  expand   the latent vectors of whole requests become keys and values of all heads: a product with the layer's weights, rows from pages
  prefill  chunks of new tokens attend to expanded keys and values, causally

Lists of lengths are texts ("811,328"): one entry per request.
"""
import math

import torch

own = False

DEV = "cuda:0"
PAGE = 16
ROPE = 64
EPS = 1e-6
BASE = 10000.0
BF16 = torch.bfloat16


def _ints(text):
    return [int(x) for x in text.split(",")]


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _spread(n, low, high, step):
    """n lengths between low and high, spread over their logarithm in an order that is not sorted."""
    return [round(low * (high / low) ** ((i * step % n + 0.5) / n)) for i in range(n)]


def listed():
    return [
        # the second half of a 16k prompt, one layer, 16 heads of a model that is spread over eight GPUs
        dict(name="append_prompt_8k", kind="append", form="prompt", heads=16, latent=512, head_dim=128, layout="pairs", norm=True, prefix="8192", new="8192"),
        # a mixed batch of chunks behind cached prefixes, all 128 heads on one GPU
        dict(name="append_mixed_batch", kind="append", form="prompt", heads=128, latent=512, head_dim=128, layout="half", norm=True,
             prefix=_text(_spread(16, 60, 60000, 7)), new=_text(_spread(16, 30, 900, 5))),
        # the smallest calls: a decode step of 64 requests at positions up to 100k
        dict(name="append_tokens_64", kind="append", form="tokens", tokens=1, heads=16, latent=512, head_dim=128, layout="pairs", norm=True,
             lens=_text(_spread(64, 30, 100000, 27))),
        # one question behind a 128k document, 16 heads: everything is the cache's bytes
        dict(name="absorb_one_128k", kind="absorb", tokens=1, heads=16, latent=512, head_dim=128, lens="131071"),
        # an ordinary serving batch with all 128 heads on one GPU: 48 requests of uneven length and three padding rows of a captured batch
        dict(name="absorb_batch_51", kind="absorb", tokens=1, heads=128, latent=512, head_dim=128, lens=_text(_spread(48, 120, 8000, 29)) + ",0,0,0"),
        # drafted tokens to be verified: four a row, 16 heads
        dict(name="absorb_drafts_64", kind="absorb", tokens=4, heads=16, latent=512, head_dim=128, lens=_text(_spread(64, 40, 6000, 27))),
        # the smallest call: four requests of a small model, one of them at its first token
        dict(name="absorb_tiny", kind="absorb", tokens=1, heads=10, latent=256, head_dim=64, lens="1,17,300,1000"),
        # the keys and values of a 128k document, 16 heads of 128
        dict(name="expand_128k", kind="expand", heads=16, latent=512, head_dim=128, lens="131072"),
        # a short batch of a small model
        dict(name="expand_small", kind="expand", heads=10, latent=256, head_dim=64, lens="77,1003,5,340"),
        # the second half of a 16k prompt
        dict(name="prefill_8k_8k", kind="prefill", heads=16, head_dim=128, latent=512, prefix="8192", new="8192"),
        # a mixed batch of chunks behind prefixes that were reused
        dict(name="prefill_mixed_batch", kind="prefill", heads=16, head_dim=128, latent=512, prefix=_text(_spread(8, 60, 9000, 3)),
             new=_text(_spread(8, 90, 2500, 5))),
        # a short follow-up question of a small model behind a long prefix
        dict(name="prefill_short_chunk", kind="prefill", heads=10, head_dim=64, latent=256, prefix="20011", new="45"),
    ]


def draw(rng):
    def log(low, high):
        return int(round(low * (high / low) ** rng.random()))

    kind = rng.choice(("append", "absorb", "absorb", "expand", "prefill"))
    head_dim, latent = rng.choice(((128, 512), (128, 512), (64, 256), (64, 512), (128, 256)))
    shape = dict(kind=kind, heads=rng.choice((1, 5, 8, 10, 16, 16, 32, 40, 64, 128)), latent=latent, head_dim=head_dim)
    if kind == "append":
        extra = dict(shape, layout=rng.choice(("half", "pairs")), norm=rng.random() < 0.7)
        if rng.random() < 0.5:
            tokens = rng.choice((1, 1, 1, 2, 4))
            return dict(extra, form="tokens", tokens=tokens, lens=_text(log(tokens, 100000) for _ in range(log(1, 200))))
        n = log(1, 40)
        most = 4096 * 128 // shape["heads"] // n
        return dict(extra, form="prompt", prefix=_text(log(1, 60000 // n + 2) - 1 for _ in range(n)),
                    new=_text(log(1, min(8192, max(2, most))) for _ in range(n)))
    if kind == "absorb":
        n, tokens = log(1, 160), rng.choice((1, 1, 1, 2, 4))
        # (padded to its longest request, a case has no more scores than a batch of 51 requests of 8000 with 128 heads, and no more keys)
        longest = log(tokens, max(2 * tokens, min(131071, 408000 // n, 51 * 8000 * 128 // (n * shape["heads"] * tokens))))
        return dict(shape, tokens=tokens, lens=_text(0 if rng.random() < 0.04 else log(tokens, longest) for _ in range(n - 1)) + ("," if n > 1 else "") + str(longest))
    if kind == "expand":
        n = log(1, 30)
        most = 131072 * 16 * 128 // (shape["heads"] * head_dim) // n
        return dict(shape, lens=_text(log(1, max(2, min(131072 // n, most))) for _ in range(n)))
    n = log(1, 12)
    chunk = log(1, min(8192, max(2, 20000 // n)))
    keys = max(chunk + 1, min(60000 // n, 16 * 8192 * 8192 // (n * shape["heads"] * chunk)))
    prefix = [log(1, keys - chunk + 1) - 1 for _ in range(n)]
    return dict(shape, heads=min(shape["heads"], max(1, 16 * 8192 * 8192 // (n * chunk * keys))), prefix=_text(prefix), new=_text([log(1, chunk) for _ in range(n - 1)] + [chunk]))


# ---- inputs ----

def _tables(lens, gen, before=None):
    """Pages of the requests scattered over a pool that has a few more: (block tables, pages in the pool).  The first
    ``before`` tokens of a request lie in pages that all of them share."""
    skip = [0] * len(lens) if before is None else [n // PAGE for n in before]
    need = [-(-n // PAGE) - k for n, k in zip(lens, skip)]
    pool, wide = sum(need) + 7, max(1, max(n + k for n, k in zip(need, skip)))
    ids = torch.randperm(pool, device=DEV, generator=gen).to(torch.int32)
    starts = torch.tensor([7 + sum(need[:r]) - skip[r] for r in range(len(lens))], device=DEV)
    column = torch.arange(wide, device=DEV)
    at = torch.where(column < torch.tensor(skip, device=DEV)[:, None], column % 7, (starts[:, None] + column).clamp(0, pool - 1))
    return ids[at].contiguous(), pool


def _random(shape, gen):
    return torch.randn(shape, device=DEV, generator=gen, dtype=BF16)


def _of_rows(values):
    return torch.tensor(values, device=DEV)


def _inputs_append(case, gen):
    H, R, D = case["heads"], case["latent"], case["head_dim"]
    if case["form"] == "tokens":
        lens = _ints(case["lens"])
        new = [case["tokens"]] * len(lens)
        prefix = [n - case["tokens"] for n in lens]
    else:
        prefix, new = _ints(case["prefix"]), _ints(case["new"])
        lens = [p + c for p, c in zip(prefix, new)]
    tables, pages = _tables(lens, gen, prefix)
    T = sum(new)
    s = dict(case=case, tables=tables, pages=pages, prefix=prefix, new=new, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    # the query's rotated columns stand behind its others in every head; what is rotated goes to the place the next step reads it from
    # (behind the absorbed columns of a decode step, as it stood in a prompt)
    s["q"] = _random((T, H, D + ROPE), gen)[:, :, D:]
    at = R if case["form"] == "tokens" else D
    s["q_out"] = torch.zeros((T, H, at + ROPE), dtype=BF16, device=DEV)[:, :, at:]
    s["kv"] = _random((T, R + ROPE), gen)
    s["norm"] = (1 + 0.1 * torch.randn((R,), device=DEV, generator=gen)).to(BF16) if case["norm"] else None
    s["inv_freq"] = BASE ** (-torch.arange(0, ROPE, 2, dtype=torch.float64, device=DEV) / ROPE)
    s["row_of"] = torch.repeat_interleave(torch.arange(len(new), device=DEV), _of_rows(new))
    first = _of_rows([p - sum(new[:r]) for r, p in enumerate(prefix)])
    s["position"] = first[s["row_of"]] + torch.arange(T, device=DEV)
    s["pool"] = torch.zeros((pages, PAGE, R + ROPE), dtype=BF16, device=DEV)
    s["scratch"] = torch.empty(64 + 32 * len(new), dtype=torch.uint8, device=DEV)
    return s


def _inputs_absorb(case, gen):
    H, R, n, lens = case["heads"], case["latent"], case["tokens"], _ints(case["lens"])
    tables, pages = _tables(lens, gen)
    rows = len(lens) * n
    return dict(case=case, tables=tables, pages=pages, lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                q=_random((rows, H, R + ROPE), gen), pool=_random((pages, PAGE, R + ROPE), gen),
                out=torch.zeros((rows, H, R), dtype=BF16, device=DEV), lse=torch.zeros((rows, H), device=DEV))


def _places(tables, lens):
    """Page and slot of every token of whole requests, requests back to back."""
    row = torch.repeat_interleave(torch.arange(len(lens), device=DEV), _of_rows(lens))
    at = torch.arange(sum(lens), device=DEV) - _of_rows([sum(lens[:r]) for r in range(len(lens))])[row]
    return tables[row, at // PAGE].long(), at % PAGE


def _inputs_expand(case, gen):
    H, R, D, lens = case["heads"], case["latent"], case["head_dim"], _ints(case["lens"])
    tables, pages = _tables(lens, gen)
    s = dict(case=case, tables=tables, pages=pages, list=lens, pool=_random((pages, PAGE, R + ROPE), gen),
             weight=(torch.randn((H * 2 * D, R), device=DEV, generator=gen) / math.sqrt(R)).to(BF16),
             kv=torch.zeros((sum(lens), H, 2 * D), dtype=BF16, device=DEV), scratch=torch.empty(64 + 32 * len(lens), dtype=torch.uint8, device=DEV))
    s["page"], s["slot"] = _places(tables, lens)
    return s


def _inputs_prefill(case, gen):
    H, R, D, prefix, new = case["heads"], case["latent"], case["head_dim"], _ints(case["prefix"]), _ints(case["new"])
    lens = [p + c for p, c in zip(prefix, new)]
    tables, pages = _tables(lens, gen)
    T, N, n = sum(new), sum(lens), len(lens)
    s = dict(case=case, tables=tables, pages=pages, prefix=prefix, new=new, pool=_random((pages, PAGE, R + ROPE), gen),
             q=_random((T, H, D + ROPE), gen), kv=_random((N, H, 2 * D), gen), out=torch.zeros((T, H, D), dtype=BF16, device=DEV),
             lse=torch.zeros((T, H), device=DEV))
    s["k"], s["v"] = s["kv"][:, :, :D], s["kv"][:, :, D:]
    # places of a padded batch: token i of request r, or its last one where it has fewer
    def padded(sizes):
        sizes, starts = _of_rows(sizes), _of_rows([sum(sizes[:r]) for r in range(n)])
        i = torch.arange(int(sizes.max()), device=DEV)
        return starts[:, None] + torch.minimum(i, sizes[:, None] - 1), i < sizes[:, None]
    s["q_at"], s["q_in"] = padded(new)
    s["k_at"], s["k_in"] = padded(lens)
    s["page"], s["slot"] = _places(tables, lens)
    s["starts"] = _of_rows(prefix)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    make = dict(append=_inputs_append, absorb=_inputs_absorb, expand=_inputs_expand, prefill=_inputs_prefill)[case["kind"]]
    return make(case, gen)


# ---- the plain forms: elementary operations in 32 bits ----

def _plain_append(s):
    c = s["case"]
    R = c["latent"]
    angle = s["position"].double()[:, None] * s["inv_freq"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turned(x, cos, sin):
        if c["layout"] == "half":
            u, v = x[..., : ROPE // 2], x[..., ROPE // 2:]
            return torch.cat((u * cos - v * sin, v * cos + u * sin), -1)
        u, v = x[..., 0::2], x[..., 1::2]
        return torch.stack((u * cos - v * sin, v * cos + u * sin), -1).flatten(-2)

    s["q_out"].copy_(turned(s["q"].float(), cos[:, None], sin[:, None]).to(BF16))
    x = s["kv"].float()
    latent = x[:, :R]
    if s["norm"] is not None:
        latent = latent * torch.rsqrt((latent * latent).mean(-1, keepdim=True) + EPS) * s["norm"].float()
    row = torch.cat((latent, turned(x[:, R:], cos, sin)), -1)
    s["pool"][s["tables"][s["row_of"], s["position"] // PAGE].long(), s["position"] % PAGE] = row.to(BF16)
    return s["q_out"], s["pool"]


def _softmax_of(x, v):
    """(softmax(x) v, log-sum-exp of x) over the last axis of x; rows that see nothing give 0 and -inf."""
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total), (top + torch.log(total))[..., 0]


def _plain_absorb(s):
    c = s["case"]
    H, R, n, B = c["heads"], c["latent"], c["tokens"], s["lens"].shape[0]
    keys = s["pool"][s["tables"].long()].reshape(B, -1, R + ROPE).float()
    # row t H + h of a request sees the keys before len - n + t + 1
    limit = s["lens"][:, None] - n + 1 + torch.arange(n, device=DEV)
    limit = torch.where(s["lens"][:, None] > 0, limit, torch.zeros_like(limit)).repeat_interleave(H, 1)
    x = torch.matmul(s["q"].float().reshape(B, n * H, R + ROPE), keys.transpose(1, 2)) / math.sqrt(c["head_dim"] + ROPE)
    x = x.masked_fill(torch.arange(keys.shape[1], device=DEV) >= limit[..., None], -math.inf)
    out, lse = _softmax_of(x, keys[..., :R])
    s["out"].copy_(out.reshape(B * n, H, R).to(BF16))
    s["lse"].copy_(lse.reshape(B * n, H))
    return s["out"], s["lse"]


def _plain_expand(s):
    rows = s["pool"][s["page"], s["slot"], : s["case"]["latent"]].float()
    s["kv"].copy_(torch.matmul(rows, s["weight"].float().t()).to(BF16).view(s["kv"].shape))
    return s["kv"]


def _plain_prefill(s):
    D = s["case"]["head_dim"]
    shared = s["pool"][s["page"], s["slot"], s["case"]["latent"]:].float()[s["k_at"]]              # [B, keys, ROPE]
    q, k, v = (s[name].float()[s[at]].transpose(1, 2) for name, at in (("q", "q_at"), ("k", "k_at"), ("v", "k_at")))
    x = (torch.matmul(q[..., :D], k.transpose(2, 3)) + torch.matmul(q[..., D:], shared[:, None].transpose(2, 3))) / math.sqrt(D + ROPE)
    i, j = torch.arange(q.shape[2], device=DEV), torch.arange(k.shape[2], device=DEV)
    seen = (j <= (s["starts"][:, None] + i)[..., None]) & s["k_in"][:, None]
    out, lse = _softmax_of(x.masked_fill_(~seen[:, None], -math.inf), v)
    s["out"].copy_(out.transpose(1, 2)[s["q_in"]].to(BF16))
    s["lse"].copy_(lse.transpose(1, 2)[s["q_in"]])
    return s["out"], s["lse"]


# ---- the framework's calls ----

def _kept(s, name, make):
    """What a program makes once and keeps beside its inputs."""
    if name not in s:
        s[name] = make()
    return s[name]


def _params(s):
    from paper_2407_00079_amd import binding as B
    c = s["case"]
    return _kept(s, "params", lambda: B.latent_params(c["heads"], c["latent"], ROPE, c["head_dim"], PAGE, s["pages"], "bf16"))


def _own_append(s):
    from paper_2407_00079_amd import binding as B
    c, p = s["case"], _params(s)
    rope = _kept(s, "rope", lambda: B.rope_params(ROPE, B.MC_ROPE_HALF if c["layout"] == "half" else B.MC_ROPE_PAIRS, base=BASE, norm_eps=EPS))
    if c["form"] == "tokens":
        B.mc_latent_append_decode(p, rope, s["q"], s["kv"], s["norm"], s["q_out"], s["pool"], s["tables"], s["lens"], c["tokens"])
    else:
        B.mc_latent_append_paged(p, rope, s["q"], s["kv"], s["norm"], s["q_out"], s["pool"], s["tables"], s["prefix"], s["new"], s["scratch"])
    return s["q_out"], s["pool"]


def _own_absorb(s):
    from paper_2407_00079_amd import binding as B
    p, n = _params(s), s["case"]["tokens"]
    work = _kept(s, "work", lambda: torch.empty(B.mc_latent_decode_attn_workspace_bytes(p, s["lens"].shape[0], n), dtype=torch.uint8, device=DEV))
    B.mc_latent_decode_attn_paged(p, s["q"], s["pool"], s["tables"], s["lens"], n, s["out"], s["lse"], work)
    return s["out"], s["lse"]


def _own_expand(s):
    from paper_2407_00079_amd import binding as B
    B.mc_latent_expand_paged(_params(s), s["weight"], s["pool"], s["tables"], s["list"], s["kv"], s["scratch"])
    return s["kv"]


def _own_prefill(s):
    from paper_2407_00079_amd import binding as B
    p = _params(s)
    work = _kept(s, "work", lambda: torch.empty(B.mc_latent_prefill_attn_workspace_bytes(p, s["prefix"], s["new"]), dtype=torch.uint8, device=DEV))
    B.mc_latent_prefill_attn_paged(p, s["q"], s["k"], s["v"], s["pool"], s["tables"], s["prefix"], s["new"], s["out"], s["lse"], work)
    return s["out"], s["lse"]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return dict(append=_own_append, absorb=_own_absorb, expand=_own_expand, prefill=_own_prefill)[kind](state)
    return dict(append=_plain_append, absorb=_plain_absorb, expand=_plain_expand, prefill=_plain_prefill)[kind](state)


# ---- what a pass cannot do without ----

def work(case):
    H, R, D = case["heads"], case["latent"], case["head_dim"]
    if case["kind"] == "append":
        T = len(_ints(case["lens"])) * case["tokens"] if case["form"] == "tokens" else sum(_ints(case["new"]))
        return dict(bytes=2 * 2 * T * (H * ROPE + R + ROPE), flops=T * (3 * ROPE * (H + 1) + 4 * R * case["norm"]))
    if case["kind"] == "absorb":
        lens, n = _ints(case["lens"]), case["tokens"]
        seen = sum(max(0, k - n + 1 + t) for k in lens if k > 0 for t in range(n))
        rows = len(lens) * n * H
        return dict(bytes=2 * sum(lens) * (R + ROPE) + 2 * rows * (2 * R + ROPE) + 4 * rows, flops=2 * H * (2 * R + ROPE) * seen)
    if case["kind"] == "expand":
        N = sum(_ints(case["lens"]))
        return dict(bytes=2 * (N * R + H * 2 * D * R + N * H * 2 * D), flops=2 * N * R * H * 2 * D)
    prefix, new = _ints(case["prefix"]), _ints(case["new"])
    T, N = sum(new), sum(prefix) + sum(new)
    seen = sum(c * p + c * (c + 1) // 2 for p, c in zip(prefix, new))
    return dict(bytes=2 * (N * H * 2 * D + N * ROPE + T * H * (2 * D + ROPE)) + 4 * T * H, flops=2 * H * (2 * D + ROPE) * seen)


# ---- the definitions in 64 bits ----

def _rows_of(s, r, n):
    """The first n cache rows of request r in 64 bits."""
    return s["pool"][s["tables"][r, : -(-n // PAGE)].long()].flatten(0, 1)[:n].double()


def exact(case, seed):
    s = prepare(case, seed)
    H, R, D = case["heads"], case["latent"], case["head_dim"]
    scale = (D + ROPE) ** -0.5
    if case["kind"] == "append":
        turn = torch.exp(1j * s["position"][:, None].double() * s["inv_freq"])
        first = torch.arange(ROPE // 2, device=DEV) if case["layout"] == "half" else 2 * torch.arange(ROPE // 2, device=DEV)
        second = first + (ROPE // 2 if case["layout"] == "half" else 1)

        def turned(x):
            z = torch.complex(x[:, first], x[:, second]) * turn
            y = torch.empty_like(x)
            y[:, first], y[:, second] = z.real, z.imag
            return y

        q_out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        for h in range(H):
            q_out[:, h] = turned(s["q"][:, h].double())
        pool = torch.zeros(s["pool"].shape, dtype=torch.float64, device=DEV)
        x = s["kv"].double()
        latent = x[:, :R]
        if s["norm"] is not None:
            latent = latent / torch.sqrt((latent ** 2).sum(1, keepdim=True) / R + EPS) * s["norm"].double()
        page, slot = s["tables"][s["row_of"], s["position"] // PAGE].long(), s["position"] % PAGE
        pool[page, slot, :R], pool[page, slot, R:] = latent, turned(x[:, R:])
        return q_out, pool
    if case["kind"] == "absorb":
        n = case["tokens"]
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
        for r, length in enumerate(_ints(case["lens"])):
            if length == 0:
                continue
            rows = _rows_of(s, r, length)
            for t in range(n):
                seen = length - n + 1 + t
                if seen > 0:
                    score = (s["q"][r * n + t].double() @ rows[:seen].T) * scale
                    lse[r * n + t] = torch.logsumexp(score, 1)
                    out[r * n + t] = torch.softmax(score, 1) @ rows[:seen, :R]
        return out, lse
    if case["kind"] == "expand":
        w = s["weight"].double().T.contiguous()
        parts = [_rows_of(s, r, n)[:, :R] @ w for r, n in enumerate(_ints(case["lens"]))]
        return torch.cat(parts).view(s["kv"].shape)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    t0 = n0 = 0
    for r, (p, c) in enumerate(zip(s["prefix"], s["new"])):
        shared = _rows_of(s, r, p + c)[:, R:]
        hidden = torch.arange(p + c, device=DEV) > p + torch.arange(c, device=DEV)[:, None]
        for h in range(H):
            key = torch.cat((s["k"][n0: n0 + p + c, h].double(), shared), 1)
            score = ((s["q"][t0: t0 + c, h].double() @ key.T) * scale).masked_fill_(hidden, -math.inf)
            lse[t0: t0 + c, h] = torch.logsumexp(score, 1)
            out[t0: t0 + c, h] = torch.softmax(score, 1) @ s["v"][n0: n0 + p + c, h].double()
        t0, n0 = t0 + c, n0 + p + c
    return out, lse
