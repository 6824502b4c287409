"""Expansion with as many tiles of tokens as each XCD takes some of its own, outputs by groups of eight tiles: the last group smaller, the tiles of tokens no
multiple of the XCDs.  Every row is compared."""
import pytest

from test_gpu_latent_prefill import test_expand as expands

pytestmark = pytest.mark.gpu


# tiles of tokens by tiles of outputs: 65 of 128 tokens by 5, 11 and 2; 66 of 256 by 18, 65 by 15, 260 by 5
@pytest.mark.parametrize("latent,head_dim,heads,lens", [
    (256, 64, 10, [8000, 0, 1, 299]), (512, 128, 11, [100] * 83), (512, 64, 3, [8193]), (512, 128, 18, [16000, 700, 1]), (512, 128, 15, [5, 16500]),
    (256, 64, 10, [40000, 26400])])
def test_every_row(latent, head_dim, heads, lens):
    expands(latent, head_dim, heads, lens)
