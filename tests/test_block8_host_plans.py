"""How products of given sizes are done (no GPU): the sizes that the tests on a GPU take still reach every way."""
import random

import pytest

from block8_plans import EVERY, SIZES
from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import block8 as K


@pytest.mark.parametrize("gated,tile,split,rows,k,n", EVERY)
def test_sizes_of_the_gpu_tests_go_the_way_they_are_there_for(gated, tile, split, rows, k, n):
    assert K.d3_matmul8_plan(rows, n, k, gated) == (tile, split)


def test_there_is_no_way_without_a_size():
    rng = random.Random(1)
    ways = set()
    for _ in range(60000):
        rows, n, k = (int(2 ** rng.uniform(0, top)) for top in (13.5, 15, 11))
        gated = rng.randrange(2)
        ways.add((gated, *K.d3_matmul8_plan(rows, n, 16 * k, gated)))
    assert ways <= set(SIZES), ways - set(SIZES)


@pytest.mark.parametrize("rows,n,k,gated", [(0, 1, 16, 0), (-1, 1, 16, 0), (2 ** 31 - 1, 1, 16, 0), (1, 0, 16, 0), (1, 1, 0, 0), (1, 1, 24, 0)])
def test_plans_that_are_refused(rows, n, k, gated):
    with pytest.raises(B.D3Error) as e:
        K.d3_matmul8_plan(rows, n, k, gated)
    assert e.value.code == B.EINVAL
    assert B.LIB.d3_matmul8_plan(1, 1, 16, 0, None) == B.EINVAL and B.LIB.d3_matmul8_plan(1, 1, 16, 2, (B.C.c_int32 * 2)()) == B.EINVAL
