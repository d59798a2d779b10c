"""silu(gate) * up where exp(-gate) is next to the largest number: the quotient is small, but a normal number as far as exp(-gate) is finite."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
BF16, FP32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn

# gates as (a number of e4m3, a scale of few bits): their products are exact
GATES = [(-88.0, 1 - 2.0 ** -7), (-88.0, 1.0), (-88.0, 1 + 2.0 ** -7), (-44.0, 2.0), (-80.0, 1.09375), (-80.0, 1.1015625), (-96.0, 0.92), (-96.0, 1.0), (-88.0, 16.0),
         (-80.0, 1.0), (-16.0, 1.0), (-1.0, 1.0), (0.0, 1.0), (1.0, 1.0), (16.0, 1.0), (88.0, 1.0), (96.0, 16.0)]


@pytest.mark.parametrize("rows,n", [(1, 128), (20, 128), (50, 128), (100, 128), (600, 4096)])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 100])
def test_gates_whose_exponential_is_next_to_the_largest_number(rows, n, size):
    """A row's only number is 1, so both sums are single products without an error, and what is left is silu's own: exp takes an error of 2^-22 in
    the exponential unit, 2^-24 in its correction and 2^-24 in the sum with 1; the reciprocal 2^-23; the two products 2^-24 each: 10 of 2^-24.
    The correction's own argument is rounded, to 2^-24 of at most 2^-18, and its second order is below 2^-36: 1 more of 2^-24 for both."""
    k = 16
    a = torch.zeros((rows, k), device="cuda")
    a[:, 0] = 1.0
    one = torch.ones((rows, 1), device="cuda")
    for e4m3, scale in GATES:
        gq, uq = (torch.zeros((n, k), device="cuda") for _ in range(2))
        gq[:, 0] = e4m3
        uq[:, 0] = torch.arange(n, device="cuda") % 7 - 3.0
        blocks = F.blocks(n)
        gs, us = torch.full((blocks, 1), scale, device="cuda"), torch.full((blocks, 1), size, device="cuda")
        out, _ = K.d3_gated_matmul8(a.to(E4M3), one, K.Weight8(gq.to(E4M3), gs), K.Weight8(uq.to(E4M3), us), dtype=FP32)
        g = (e4m3 * gs[0, 0]).double().cpu()               # (one rounding to fp32 where the scale has more bits: the kernel's own)
        u = (uq[:, 0].double() * size).cpu()
        if float(-g) > 88.7228:                            # exp(-gate) is above the largest number: 0
            assert (out == 0).all(), (e4m3, scale)
            continue
        want = (g / (1 + torch.exp(-g)) * u).expand(rows, n)
        off, near = (out.double().cpu() - want).abs(), want.abs() * (11 * 2.0 ** -24) + 2.0 ** -149
        assert (off <= near).all(), (e4m3, scale, float((off / near).max()))
