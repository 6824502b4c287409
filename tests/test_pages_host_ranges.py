"""Numbers of rows and lengths of lists that the page kernels' 32-bit counters do not hold are refused on the host."""
import pytest

from paper_2407_00079_amd import binding as B
from test_pages_host import call


@pytest.mark.parametrize("form", ["fork", "grow", "free", "remap"])
@pytest.mark.parametrize("rows", [2 ** 30, 2 ** 31 - 1024, 2 ** 31 - 1])
@pytest.mark.parametrize("wide", [0, 1])
def test_rows(form, rows, wide):
    assert call(form, rows=rows, wide=wide, ws_bytes=2 ** 40) == B.MC_ERR_RANGE


@pytest.mark.parametrize("n", [2 ** 30, 2 ** 31 - 1])
def test_rows_to_free(n):
    assert call("free", n=n) == B.MC_ERR_RANGE and call("free", n=n, wide=0) == B.MC_ERR_RANGE


def test_workspace_of_what_is_refused():
    assert B.mc_kv_pages_workspace_bytes(64, 2 ** 30) == 0 and B.mc_kv_pages_workspace_bytes(64, 2 ** 30 - 1) > 12 * (2 ** 30 - 1)
