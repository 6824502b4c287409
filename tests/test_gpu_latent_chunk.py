"""A chunk of new tokens in the absorbed form, 16 of them a row: rows of one block table line, each as long as its last token's position says."""
import pytest
import torch

from latent_util import BF16, DEV, P, absorbed_reference, assert_near, gen, lens_tensor, params, randn, tables, workspace
from paper_2407_00079_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,latent,head_dim", [(16, 512, 128), (10, 256, 64), (128, 512, 128)])
@pytest.mark.parametrize("prefix,chunk", [(500, 40), (0, 16), (1000, 100), (7, 33)])
def test_chunk_by_rows(heads, latent, head_dim, prefix, chunk):
    g, n = gen(prefix + heads), prefix + chunk
    line, pages = tables(g, [n])
    p, rope = params(heads, latent, head_dim, pages), B.rope_params(P, B.MC_ROPE_PAIRS)
    pool, down = randn(g, pages, 16, latent + P), randn(g, chunk, latent + P)
    q_all = randn(g, chunk, heads, latent + P)
    turned, plain = q_all[:, :, latent:], q_all[:, :, latent:].clone()
    B.mc_latent_append_paged(p, rope, plain, down, None, turned, pool, line, [prefix], [chunk], workspace(B.mc_latent_workspace_bytes(1)))
    # whole rows of 16, then the last tokens as a row of so many
    whole, out, lse = chunk // 16, torch.full((chunk, heads, latent), 7.0, dtype=BF16, device=DEV), torch.full((chunk, heads), 7.0, device=DEV)
    for rows, tokens, at, lens in ((whole, 16, 0, [prefix + 16 * (i + 1) for i in range(whole)]), (1, chunk % 16, 16 * whole, [n])):
        if rows * tokens == 0:
            continue
        part = slice(at, at + rows * tokens)
        ws = workspace(B.mc_latent_decode_attn_workspace_bytes(p, rows, tokens))
        B.mc_latent_decode_attn_paged(p, q_all[part], pool, line.expand(rows, -1).contiguous(), lens_tensor(lens), tokens, out[part], lse[part], ws)
    want, want_lse, out_off, lse_off = absorbed_reference(q_all, pool, line, [n], chunk, latent, (head_dim + P) ** -0.5)
    assert_near(lse, want_lse, lse_off, "lse")
    assert_near(out, want, out_off, "out")
