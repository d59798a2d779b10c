"""Host side of the 8-bit products at the ends of their sizes (no GPU): what is next to 2^31 is refused, since the tiles' last rows lie beyond it."""
import ctypes as C

import pytest

from paper_2503_08524_b200 import binding as B
from test_block8_host import BF16, E4M3, FAKE, MB, product_args, weight

MOST = 2 ** 31 - 256


@pytest.mark.parametrize("rows,n,k", [(2 ** 31 - 1, 1, 16), (MOST + 1, 1, 16), (1, 2 ** 31 - 1, 16), (1, MOST + 1, 16), (1, 1, 2 ** 31 - 16), (1, 1, MOST + 16)])
def test_sizes_next_to_two_to_the_31_are_refused(rows, n, k):
    far = FAKE << 12                                     # (every buffer far from every other)
    w = weight(n=n, k=k, row_stride=k, q_dev=2 * far, scale_dev=3 * far)
    args = product_args(n_rows=rows, a_dev=4 * far, a_scale_dev=5 * far, out_dev=6 * far, a_stride=k, a_scale_stride=-(-k // 128), out_stride=n)
    assert B.LIB.d3_matmul8(C.byref(w), C.byref(args), None) == B.EINVAL
    u = weight(n=n, k=k, row_stride=k, q_dev=7 * far, scale_dev=8 * far)
    assert B.LIB.d3_gated_matmul8(C.byref(w), C.byref(u), C.byref(args), None) == B.EINVAL
    if rows == 1:
        space = C.create_string_buffer(512)
        assert B.LIB.d3_weight8_map(C.byref(w), (C.addressof(space) + 63) & ~63) == B.EINVAL
        assert B.LIB.d3_quantize_weight(9 * far, BF16, k, C.byref(w), None) == B.EINVAL
