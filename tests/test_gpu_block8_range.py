"""Numbers in 8 bits over the whole range of their inputs' types: blocks whose largest number is above 2^126, where its reciprocal is no
normal number any more."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn

# the last top whose reciprocal is normal, the border, and what lies between it and the largest numbers
TOPS = [(FP32, 2.0 ** 126 * (1 - 2.0 ** -24)), (FP32, 2.0 ** 126), (FP32, 1.5 * 2.0 ** 126), (FP32, 2.0 ** 127), (FP32, torch.finfo(FP32).max),
        (BF16, 2.0 ** 126), (BF16, 2.0 ** 127), (BF16, torch.finfo(BF16).max)]


def large(rows, dim, top, dtype, seed=1):
    """Numbers up to `top`, which every block of 128 (of the first row on) has."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, dim), generator=g, device="cuda").clamp(-3, 3) * (top / 3)
    x[:, ::128] = top
    return x.to(dtype)


@pytest.mark.parametrize("dtype,top", TOPS)
@pytest.mark.parametrize("rows,dim", [(1, 8), (5, 504), (700, 1032)])
def test_rows_of_large_numbers(dtype, top, rows, dim):
    x = large(rows, dim, top, dtype)
    assert float(x.max()) == top
    q, s = K.d3_quantize(x)
    F.check_8_bits(q, s, x.double(), torch.zeros_like(x, dtype=torch.float64))
    half = (x.double() / 2).to(dtype)                     # (exact) and twice it: the sum is the same number
    q2, s2, total = K.d3_add_norm(half, None, add=half)
    assert torch.equal(total, x) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, s)


@pytest.mark.parametrize("dtype,top", TOPS)
def test_weights_of_large_numbers(dtype, top):
    n, k = 130, 400
    w = large(n, k, top, dtype)
    w8 = K.d3_quantize_weight(w)
    assert torch.isfinite(w8.scale).all()
    s = F.widen(w8.scale, k).repeat_interleave(128, 0)[:n]
    assert ((F.weight64(w8.q, w8.scale) - w.double()).abs() <= w.double().abs() * (2.0 ** -4 * (1 + 2.0 ** -20) + 2.0 ** -22) + s * 2.0 ** -10).all()


@pytest.mark.parametrize("rows,k,n", [(1, 256, 384), (20, 512, 300), (100, 256, 384), (600, 1024, 2000)])
def test_gated_results_of_large_numbers(rows, k, n):
    g = torch.Generator(device="cuda").manual_seed(rows)
    a, s = F.some_rows(rows, k, g)
    gate, up = F.some_weight(n, k, g), F.some_weight(n, k, g)
    gate, up = (gate[0], gate[1] * 2.0 ** 62), (up[0], up[1] * 2.0 ** 50)
    h, _ = F.gated(*F.product(a, s, *gate), *F.product(a, s, *up))
    room = torch.floor(torch.log2(torch.finfo(FP32).max / h.abs().max()) * 64) / 64 - 1 / 64        # the largest result is next to the largest number
    up = (up[0], (up[1].double() * 2.0 ** room).float())
    h, dh = F.gated(*F.product(a, s, *gate), *F.product(a, s, *up))
    assert 2.0 ** 127.9 < float(h.abs().max()) < 2.0 ** 128
    out, scale = K.d3_gated_matmul8(a, s, K.Weight8(*gate), K.Weight8(*up))
    F.check_8_bits(out, scale, h, dh)


@pytest.mark.parametrize("rows,k,n", [(1, 256, 384), (20, 512, 300), (100, 256, 384), (600, 1024, 2000)])
@pytest.mark.parametrize("power", [-40, -85, -95, -105, -120])
def test_gated_results_of_small_numbers(rows, k, n, power):
    """Down to blocks that count as 2^-100 and keep a few of their bits, or none."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    a, s = F.some_rows(rows, k, g)
    gate, up = F.some_weight(n, k, g), F.some_weight(n, k, g)
    up = (up[0], up[1] * 2.0 ** power)
    h, dh = F.gated(*F.product(a, s, *gate), *F.product(a, s, *up))
    out, scale = K.d3_gated_matmul8(a, s, K.Weight8(*gate), K.Weight8(*up))
    F.check_8_bits(out, scale, h, dh)
    if power == -120:                 # (a number of 2^-118.8 and more, half the least one's 2^-9 of that scale, is not 0)
        assert float(h.abs().max()) < 2.0 ** -100 and (scale == 2.0 ** -100 / 448).all()
    elif power >= -95:
        assert (out.float().abs().amax(1) >= 256).all()
