"""Bounded waits of the 8-bit products: a wait that nothing satisfies ends by its limit and is reported; the next call is whole."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu


@pytest.fixture
def short_waits():
    K.d3_matmul8_set_wait_ns(2_000_000)
    yield
    K.d3_matmul8_stall_next(0)
    K.d3_matmul8_set_wait_ns(2_000_000_000)


# one CTA a tile; k cut between CTAs; several row tiles; the kernel for many rows, with fewer and with more tiles than pairs of SMs
@pytest.mark.parametrize("rows,k,n", [(1, 1024, 16384), (32, 11008, 512), (128, 8192, 1024), (300, 4096, 8192), (2048, 2048, 8192)])
@pytest.mark.parametrize("gated", [False, True])
def test_a_wait_that_runs_out(short_waits, rows, k, n, gated):
    g = torch.Generator(device="cuda").manual_seed(rows)
    a = F.some_rows(rows, k, g)
    w = K.Weight8(*F.some_weight(n, k, g))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        return K.d3_gated_matmul8(*a, w, w, status=status)[0].view(torch.uint8) if gated else K.d3_matmul8(*a, w, status=status)
    want = call().clone()
    assert int(status) == 0
    K.d3_matmul8_stall_next(1)
    call()
    torch.cuda.synchronize()
    assert int(status) == B.ETIMEOUT
    status.zero_()
    assert torch.equal(call(), want) and int(status) == 0


def test_limits_and_drills_that_are_refused():
    for call, bad in ((K.d3_matmul8_set_wait_ns, 0), (K.d3_matmul8_set_wait_ns, -1), (K.d3_matmul8_stall_next, 2), (K.d3_matmul8_stall_next, -1)):
        with pytest.raises(B.D3Error):
            call(bad)
