"""Calls on a cache of latent vectors that one launch does not hold are refused as such, before anything is uploaded or launched."""
import pytest

from paper_2407_00079_amd import binding as B
from test_latent_host import call, par

MOST = 2 ** 32 - 1           # threads of a launch
APPEND, PREFILL = 256, 512   # of a workgroup


@pytest.mark.parametrize("heads", [48, 64, 1024])
def test_prefills_that_one_launch_does_not_hold(heads):
    """One workgroup a row tile and head, here of one row."""
    most = MOST // PREFILL // heads
    for n, status in ((most, B.MC_ERR_WORKSPACE), (most + 1, B.MC_ERR_RANGE)):       # (the workspace is looked at behind)
        assert call("prefill", p=par(heads=heads), prefix=(0,) * n, new=(1,) * n, max_pages=1, ws=None) == status


@pytest.mark.parametrize("heads,latent", [(1, 512), (1, 256), (16, 512), (128, 256), (1024, 512)])
def test_appends_that_one_launch_does_not_hold(heads, latent):
    """64 rotated rows a workgroup, H + 1 of a token; behind them the latent rows, 8 or 16 a workgroup."""
    def workgroups(tokens):
        return -(-tokens * (heads + 1) // 64) + -(-tokens // (8 if latent == 512 else 16))

    low, high = 1, 2 ** 31 - 1025
    while low < high:                                          # the most tokens that fit
        mid = (low + high + 1) // 2
        low, high = (mid, high) if workgroups(mid) * APPEND <= MOST else (low, mid - 1)
    p = par(heads=heads, latent=latent)
    for tokens, status in ((low, B.MC_ERR_WORKSPACE), (low + 1, B.MC_ERR_RANGE)):
        assert call("append", p=p, prefix=(0,), new=(tokens,), max_pages=2 ** 27, ws=None) == status
    assert call("append_decode", p=p, batch=low + 1, tokens=1, max_pages=1) == B.MC_ERR_RANGE
    assert call("append_decode", p=p, batch=-(-(low + 1) // 16), tokens=16, max_pages=1) == B.MC_ERR_RANGE
    # ... and every call with so few rows does fit
    assert workgroups((2 ** 30 - 192) // (heads + 9)) * APPEND <= MOST


@pytest.mark.parametrize("form", ["append", "append_decode", "decode", "expand", "prefill"])
def test_scales_past_32_bits(form):
    """The kernels take the scale times log2(e) in 32 bits: where that is infinite, 0 times it would be NaN."""
    largest = 2.0 ** 128 * (1 - 2.0 ** -25)                    # (from here on a number rounds to infinity)
    assert call(form, p=par(scale=3e38)) == B.MC_ERR_SHAPE
    assert call(form, p=par(scale=1.0001 * largest / 1.4426950408889634)) == B.MC_ERR_SHAPE
    assert call(form, p=par(scale=0.9999 * largest / 1.4426950408889634), pool=None) == B.MC_ERR_NULL     # (which is looked at behind)
