"""Calls that have nothing to look at leave the report alone, and a freed row of no valid length is emptied with all counts as they were."""
import pytest
import torch

from paper_2407_00079_amd import binding as B
from pages_util import BAD_ROW
from test_gpu_pages import DEV, ints

pytestmark = pytest.mark.gpu


def test_reports_of_calls_that_enqueue_nothing():
    counts, report, none = ints([1, 0, 0]), ints([3, 1, 4, 1]), torch.empty(0, dtype=torch.int32, device=DEV)
    ws = torch.empty(B.mc_kv_pages_workspace_bytes(3, 0), dtype=torch.uint8, device=DEV)
    B.mc_kv_pages_grow(counts, none.reshape(0, 4), 16, none, none, report, ws)
    B.mc_kv_pages_free(counts, none.reshape(0, 4), 16, none, ints([0, 5]), report)
    B.mc_kv_pages_compact(counts, none.reshape(0, 2), report, ws)
    assert report.tolist() == [3, 1, 4, 1] and counts.tolist() == [1, 0, 0]


@pytest.mark.parametrize("wide", [2, 600])
@pytest.mark.parametrize("length", [-3, 600 * 16 + 1, 2 ** 31 - 1])
def test_rows_of_no_valid_length(wide, length):
    counts, lens, report = ints([1, 1, 1, 0]), ints([length, 20, 0]), ints([9] * 4)
    tables = torch.full((3, wide), 7, dtype=torch.int32, device=DEV)
    tables[0, :2], tables[1, :2] = ints([2, 0]), ints([0, 1])
    B.mc_kv_pages_free(counts, tables, 16, lens, ints([0, 1, 0]), report)
    assert report.tolist() == [2, BAD_ROW, 0, 0] and counts.tolist() == [0, 0, 1, 0] and lens.tolist() == [0, 0, 0]
