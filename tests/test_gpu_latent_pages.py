"""Pages of latent pools through the calls that move pages of two pools at a time: two layers' pools, and a last layer's given as both."""
import pytest
import torch

from latent_util import BF16, DEV, P, PAGE, gen, randn
from paper_2407_00079_amd import binding as B

pytestmark = pytest.mark.gpu

PAGES = 300


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def pairs(layers):
    return [(layers[i], layers[min(i + 1, len(layers) - 1)]) for i in range(0, len(layers), 2)]


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("layers", [1, 2, 3, 5])
def test_moves(latent, layers):
    g, page_bytes = gen(layers), PAGE * (latent + P) * 2
    pools = [randn(g, PAGES, PAGE, latent + P) for _ in range(layers)]
    want = [x.clone() for x in pools]
    ids = torch.randperm(PAGES, device=DEV, generator=g)[:90].view(45, 2)
    ids[:, 0] = ids[:3, 0].repeat(15)                          # (a source may be in several moves)
    moves = torch.cat((ids.to(torch.int32), ints([[-1, -1]] * 5)))
    for x in want:
        x[ids[:, 1]] = x[ids[:, 0]]
    B.mc_kv_copy_pages([a for a, _ in pairs(pools)], [b for _, b in pairs(pools)], PAGES, page_bytes, moves, ints([50]))
    assert all(torch.equal(a, b) for a, b in zip(pools, want))


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("pages", [1, 7, 250])
@pytest.mark.parametrize("ordered", [False, True])
def test_store_and_load(latent, pages, ordered):
    """Layer by layer into dense buffers, through host memory, and back to other pages of fresh pools: three layers, the last one alone."""
    g, page_bytes = gen(pages), PAGE * (latent + P) * 2
    pools = [randn(g, PAGES, PAGE, latent + P) for _ in range(3)]
    ids, back = (torch.randperm(PAGES, device=DEV, generator=g)[:pages].to(torch.int32) for _ in range(2))
    fresh = [torch.full_like(x, 7.0) for x in pools]
    want = [x.clone() for x in fresh]
    for w, x in zip(want, pools):
        w[back.long()] = x[ids.long()]
    order, back_order = ints([0] * pages), ints([0] * pages)
    B.mc_kv_page_order(ids, pages, order)
    B.mc_kv_page_order(back, pages, back_order)
    packed = [torch.full((pages + 1, PAGE, latent + P), 9.0, dtype=BF16, device=DEV) for _ in range(3)]
    for (a, b), (x, y), (u, v) in zip(pairs(pools), pairs(packed), pairs(fresh)):
        if ordered:
            B.mc_kv_pack_layer_ordered(a, b, PAGES, page_bytes, ids, order, pages, x, y)
            B.mc_kv_unpack_layer_ordered(x, y, PAGES, page_bytes, back, back_order, pages, u, v)
        else:
            B.mc_kv_pack_layer(a, b, PAGES, page_bytes, ids, pages, x, y)
            B.mc_kv_unpack_layer(x, y, PAGES, page_bytes, back, pages, u, v)
    for x, y in zip(packed, pools):
        assert torch.equal(x[:pages], y[ids.long()]) and bool((x[pages] == 9).all())
    assert all(torch.equal(a, b) for a, b in zip(fresh, want))
    # the same through pinned host memory
    for x in fresh:
        x.fill_(7.0)
    held = [torch.zeros((pages, PAGE, latent + P), dtype=BF16, pin_memory=True) for _ in range(3)]
    stage = [torch.empty((pages, PAGE, latent + P), dtype=BF16, device=DEV) for _ in range(3)]
    for (a, b), (x, y), (h, i) in zip(pairs(pools), pairs(stage), pairs(held)):
        B.mc_kv_store_layer(a, b, PAGES, page_bytes, ids, pages, x, y, h, i)
    torch.cuda.synchronize()
    assert all(torch.equal(h, x[ids.long()].cpu()) for h, x in zip(held, pools))
    for (u, v), (x, y), (h, i) in zip(pairs(fresh), pairs(stage), pairs(held)):
        B.mc_kv_load_layer(h, i, x, y, PAGES, page_bytes, back, pages, u, v)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(fresh, want))
