"""Infinities in V: the definition's sums of products are infinite or, of both signs, not numbers; they are so in every form."""
import math

import pytest
import torch

from test_gpu_decode import DEV, KINDS, PAGE, Call

pytestmark = pytest.mark.gpu


def put(c, row, key, head, columns, value):
    c.v[c.table[row, key // PAGE].long(), head, key % PAGE, columns] = value


# in one wave's stretch, a workgroup's, several workgroups', and short tables (a workgroup a row)
SHAPES = [((8, 2), [700, 5000, 60]), ((8, 1), [70001, 33]), ((4, 2), [300, 17, 1]), ((40, 1), [64, 400, 9000]), ((2, 1), [45] * 600)]


@pytest.mark.parametrize("dtype,dim", KINDS)
@pytest.mark.parametrize("heads,lens", SHAPES)
def test_sums_that_are_infinite(dtype, dim, heads, lens):
    c = Call(dtype, heads, dim, lens, seed=31)
    for row, n in enumerate(lens[:3]):
        for i, key in enumerate(sorted({0, n // 3, n // 2, n - 1})):
            put(c, row, key, 0, 2 * i, math.inf)
            put(c, row, key, 0, 2 * i + 1, -math.inf)
        put(c, row, n - 1, 0, 40, math.inf)
        put(c, row, 0, 0, 40, math.inf)
        put(c, row, n - 1, 0, 41, math.nan)
        if n > 1:
            put(c, row, n - 1, 0, 42, math.inf)
            put(c, row, 0, 0, 42, -math.inf)
    c.run()
    c.check()
    seen = c.out[: min(3, len(lens))].float()
    assert bool(torch.isinf(seen).any()) and bool(torch.isnan(seen).any())


@pytest.mark.parametrize("dtype,dim", KINDS)
def test_every_key_is_infinite_in_one_column(dtype, dim):
    """Whatever p a key has (and however it is cut into parts), p times infinity is infinite."""
    c = Call(dtype, (8, 1), dim, [3001, 77], seed=32, sharp=3.0)
    for row, n in enumerate(c.lens):
        keys = torch.arange(n, device=DEV)
        c.v[c.table[row, keys // PAGE].long(), 0, keys % PAGE, 5] = math.inf
        c.v[c.table[row, keys // PAGE].long(), 0, keys % PAGE, 6] = -math.inf
    c.run()
    c.check()
    assert bool((c.out[..., 5] == math.inf).all()) and bool((c.out[..., 6] == -math.inf).all())


@pytest.mark.parametrize("dtype,dim", KINDS)
def test_equal_scores(dtype, dim):
    """p = 1 exactly for every key: nothing is left of it after its rounding."""
    c = Call(dtype, (16, 2), dim, [900, 31, 4000], seed=33)
    c.q.zero_()
    for row, n in enumerate(c.lens):
        put(c, row, n // 2, 1, 7, math.inf)
        put(c, row, n // 4, 1, 9, -math.inf)
    c.run()
    c.check()
    assert bool((c.out[:, 8:, 7] == math.inf).all()) and bool((c.out[:, 8:, 9] == -math.inf).all())
    assert int(torch.isfinite(c.out).logical_not().sum()) == 3 * 8 * 2
