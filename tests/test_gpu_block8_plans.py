"""Every way that a product can be done against 64-bit forms, with results that lie on 16 bytes and ones that do not."""
import pytest
import torch

import block8_forms as F
from block8_plans import EVERY
from paper_2503_08524_b200 import block8 as K
from test_gpu_block8 import strided

pytestmark = pytest.mark.gpu
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.mark.parametrize("gated,tile,split,rows,k,n", EVERY)
def test_every_way(gated, tile, split, rows, k, n):
    assert K.d3_matmul8_plan(rows, n, k, gated) == (tile, split)
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    a, s = F.some_rows(rows, k, g)
    weights = [F.some_weight(n, k, g) for _ in range(1 + gated)]
    y, dy = F.product(a, s, *weights[0])
    if gated:
        y, dy = F.gated(y, dy, *F.product(a, s, *weights[1]))
    handles = [K.Weight8(*w) for w in weights]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for dtype in (BF16, FP16, FP32) + ((E4M3,) if gated else ()):
        held, size = (torch.uint8, 1) if dtype is E4M3 else (dtype, dtype.itemsize)
        for extra in (0, 1, -n * size % 16 // size or 16):     # rows side by side, one number further apart, on 16 bytes each
            buf, out = strided(rows, n, held, extra)
            if dtype is E4M3:
                scales, scale = strided(rows, F.blocks(n), FP32, extra)
                K.d3_gated_matmul8(a, s, *handles, out=out.view(E4M3), scale=scale, status=status)
                F.check_8_bits(out.view(E4M3), scale, y, dy)
                scales[:rows, : F.blocks(n)] = 7
                assert (scales == 7).all()
            elif gated:
                K.d3_gated_matmul8(a, s, *handles, out=out, status=status)
                F.check_wide(out, y, dy)
            else:
                K.d3_matmul8(a, s, handles[0], out=out, status=status)
                F.check_wide(out, y, dy)
            buf[:rows, :n] = 7
            assert (buf == 7).all(), (dtype, extra)
    assert int(status) == 0
