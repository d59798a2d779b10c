"""The limit of the paged attention's waits and its drill: what the host refuses (no GPU)."""
import pytest

from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import paged as P


def test_limits_and_drills_that_are_refused():
    assert B.LIB.d3_paged_set_wait_ns(0) == B.EINVAL
    for bad in (-1, 3, 2 ** 31 - 1):
        assert B.LIB.d3_paged_stall_next(bad) == B.EINVAL
    for f, bad in ((P.d3_paged_set_wait_ns, 0), (P.d3_paged_set_wait_ns, -5), (P.d3_paged_stall_next, 7)):
        with pytest.raises(B.D3Error) as e:
            f(bad)
        assert e.value.code == B.EINVAL
    P.d3_paged_set_wait_ns(1)
    P.d3_paged_set_wait_ns(2_000_000_000)
    P.d3_paged_stall_next(P.STALL_SUMS)
    P.d3_paged_stall_next(0)
