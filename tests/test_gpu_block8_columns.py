"""Results in columns of a wider buffer: what stands beside them stays, whatever is left of the last 16 bytes of a row."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,k,n", [(217, 64, 10992), (999, 528, 4096), (1, 528, 4096), (20, 528, 640), (600, 1040, 3504)])
@pytest.mark.parametrize("less", list(range(0, 17)))
def test_columns_beside_the_results_stay(gated, rows, k, n, less):
    n -= less
    g = torch.Generator(device="cuda").manual_seed(n)
    a, s = F.some_rows(rows, k, g)
    w = [K.Weight8(*F.some_weight(n, k, g)) for _ in range(2)]
    for dtype in (BF16, FP16, FP32) + ((E4M3,) if gated else ()):
        size = 1 if dtype is E4M3 else dtype.itemsize
        width = -(-n * size // 16) * 16 + 32             # bytes: whole pieces of 16, and two more
        buf = torch.full((rows + 1, width), 0x55, dtype=torch.uint8, device="cuda")
        out = buf[:rows].view(dtype)[:, :n]
        if dtype is E4M3:
            want, _ = K.d3_gated_matmul8(a, s, *w)       # (rows side by side go another way out)
            K.d3_gated_matmul8(a, s, *w, out=out)
        elif gated:
            want, _ = K.d3_gated_matmul8(a, s, *w, dtype=dtype)
            K.d3_gated_matmul8(a, s, *w, out=out)
        else:
            want = K.d3_matmul8(a, s, w[0], dtype=dtype)
            K.d3_matmul8(a, s, w[0], out=out)
        assert torch.equal(out.float(), want.float())
        buf[:rows, : n * size] = 0x55
        assert (buf == 0x55).all(), (dtype, (buf != 0x55).nonzero()[:4].tolist())
