"""Host side of the 8-bit block operators and of the constraints on logits (no GPU): what the C ABI and the binding refuse before
anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import block8 as K

FAKE = 1 << 30        # an aligned address that no refused call may touch
MB = 1 << 20
BF16, FP16, FP32, E4M3 = 0, 1, 2, 3


def weight(**kw):
    a = K.Weight8Args(C.sizeof(K.Weight8Args), 300, 512, 512, FAKE + 64 * MB, FAKE + 65 * MB, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def norm_args(**kw):
    a = K.AddNormArgs(C.sizeof(K.AddNormArgs), 5, 256, BF16, FP32, BF16, E4M3, 1e-5, FAKE, FAKE + MB, FAKE + 2 * MB, FAKE + 3 * MB, FAKE + 4 * MB,
                      FAKE + 5 * MB, 256, 256, 256, 256, 2)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def product_args(**kw):
    a = K.Matmul8Args(C.sizeof(K.Matmul8Args), 5, BF16, FAKE, FAKE + MB, FAKE + 2 * MB, None, 512, 4, 300, 0, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def logits_args(**kw):
    p = [FAKE + (2 + i) * MB for i in range(12)]
    a = K.ConstrainLogitsArgs(C.sizeof(K.ConstrainLogitsArgs), FP32, 3, 1000, 20, 4, 2, FAKE, FAKE + MB, 1000, 1000, 20, 4, 32, *p)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(struct_size=8), dict(n_rows=-1), dict(dim=0), dict(dim=12), dict(dim=65544), dict(x_dtype=E4M3), dict(x_dtype=9), dict(add_dtype=FP16),
    dict(gain_dtype=E4M3), dict(out_dtype=7), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x_dev=None), dict(x_dev=FAKE + 8),
    dict(x_stride=252), dict(add_dev=FAKE + MB + 4), dict(add_stride=258), dict(add_dev=None), dict(total_dev=FAKE + 2 * MB + 8), dict(total_stride=128),
    dict(gain_dev=FAKE + 3 * MB + 2), dict(out_dev=None), dict(out_dev=FAKE + 4 * MB + 4), dict(out_stride=255), dict(out_stride=248), dict(scale_dev=None),
    dict(scale_stride=1), dict(scale_dev=FAKE + 5 * MB + 2), dict(out_dtype=BF16),
    # what is written overlaps something else
    dict(out_dev=FAKE + 2 * MB), dict(out_dev=FAKE), dict(scale_dev=FAKE + 4 * MB + 256), dict(total_dev=FAKE + 16), dict(total_dev=FAKE + MB + 16),
    dict(scale_dev=FAKE + 3 * MB), dict(total_dev=FAKE + MB, total_stride=512), dict(total_dev=FAKE)], ids=str)
def test_norms_that_are_refused(bad):
    assert B.LIB.d3_add_norm(C.byref(norm_args(**bad)), None) == B.EINVAL


def test_norms_without_rows_are_nothing_to_do():
    assert B.LIB.d3_add_norm(C.byref(norm_args(n_rows=0)), None) == B.OK
    assert B.LIB.d3_add_norm(None, None) == B.EINVAL


BAD_WEIGHTS = [dict(struct_size=4), dict(n=0), dict(k=0), dict(k=504), dict(row_stride=496), dict(row_stride=520), dict(q_dev=None),
               dict(q_dev=FAKE + 64 * MB + 8), dict(scale_dev=None), dict(scale_dev=FAKE + 2), dict(map=FAKE + 8)]


@pytest.mark.parametrize("bad", BAD_WEIGHTS, ids=str)
def test_weights_that_are_refused(bad):
    w, good = weight(**bad), weight()
    assert B.LIB.d3_matmul8(C.byref(w), C.byref(product_args()), None) == B.EINVAL
    assert B.LIB.d3_gated_matmul8(C.byref(good), C.byref(w), C.byref(product_args()), None) == B.EINVAL
    assert B.LIB.d3_gated_matmul8(C.byref(w), C.byref(good), C.byref(product_args()), None) == B.EINVAL
    if "map" not in bad:
        space = C.create_string_buffer(K.MAP_BYTES + 64)
        assert B.LIB.d3_weight8_map(C.byref(w), (C.addressof(space) + 63) & ~63) == B.EINVAL
        assert B.LIB.d3_quantize_weight(FAKE, BF16, 512, C.byref(w), None) == B.EINVAL


@pytest.mark.parametrize("bad", [
    dict(struct_size=0), dict(n_rows=-1), dict(out_dtype=E4M3), dict(out_dtype=5), dict(a_dev=None), dict(a_dev=FAKE + 8), dict(a_scale_dev=None),
    dict(a_scale_dev=FAKE + 1), dict(out_dev=None), dict(out_dev=FAKE + 2 * MB + 1), dict(a_stride=496), dict(a_stride=520), dict(a_scale_stride=3),
    dict(out_stride=299), dict(scale_dev=FAKE + 3 * MB), dict(status_dev=FAKE + 2), dict(out_dev=FAKE + 16), dict(out_dev=FAKE + MB),
    dict(out_dev=FAKE + 64 * MB), dict(out_dev=FAKE + 65 * MB), dict(status_dev=FAKE + 2 * MB), dict(status_dev=FAKE)], ids=str)
def test_products_that_are_refused(bad):
    assert B.LIB.d3_matmul8(C.byref(weight()), C.byref(product_args(**bad)), None) == B.EINVAL


@pytest.mark.parametrize("bad", [dict(scale_dev=None), dict(scale_stride=2), dict(scale_dev=FAKE + 2 * MB), dict(scale_dev=FAKE), dict(scale_dev=FAKE + 3 * MB + 2)],
                         ids=str)
def test_gated_products_that_are_refused(bad):
    args = dict(out_dtype=E4M3, scale_dev=FAKE + 3 * MB, scale_stride=3)
    args.update(bad)
    w = weight()
    assert B.LIB.d3_gated_matmul8(C.byref(w), C.byref(weight()), C.byref(product_args(**args)), None) == B.EINVAL
    assert B.LIB.d3_gated_matmul8(C.byref(w), C.byref(weight(n=299)), C.byref(product_args()), None) == B.EINVAL
    assert B.LIB.d3_gated_matmul8(C.byref(w), C.byref(weight(k=496)), C.byref(product_args()), None) == B.EINVAL
    assert B.LIB.d3_gated_matmul8(C.byref(w), None, C.byref(product_args()), None) == B.EINVAL


def test_products_without_rows_are_nothing_to_do():
    assert B.LIB.d3_matmul8(C.byref(weight()), C.byref(product_args(n_rows=0)), None) == B.OK


@pytest.mark.parametrize("dtype,stride,at", [(E4M3, 512, FAKE), (7, 512, FAKE), (BF16, 511, FAKE), (BF16, 512, None), (BF16, 512, FAKE + 1),
                                             (BF16, 512, FAKE + 64 * MB + 16), (FP32, 512, FAKE + 65 * MB)])
def test_weights_that_are_not_quantized(dtype, stride, at):
    assert B.LIB.d3_quantize_weight(at, dtype, stride, C.byref(weight()), None) == B.EINVAL


@pytest.mark.parametrize("bad", [
    dict(struct_size=1), dict(dtype=E4M3), dict(n_rows=-1), dict(n_rows=65536), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(n_history=-1), dict(n_bias=-1), dict(n_history=(1 << 30) + 1), dict(n_bias=(1 << 30) + 1),
    dict(n_masks=-1), dict(logits_dev=None), dict(out_dev=None), dict(logits_dev=FAKE + 2), dict(out_dev=FAKE + MB + 1), dict(out_stride=999),
    dict(history_dev=None), dict(bias_dev=None), dict(bias_ids_dev=None), dict(masks_dev=None), dict(mask_of_dev=None), dict(history_stride=-1),
    dict(bias_stride=-4), dict(mask_stride=-1), dict(token_dev=FAKE + 2), dict(status_dev=FAKE + 3), dict(lengths_dev=FAKE + 1),
    dict(out_dev=FAKE + 4), dict(out_dev=FAKE, out_stride=1004), dict(token_dev=FAKE), dict(token_dev=FAKE + MB), dict(token_dev=FAKE + 2 * MB),
    dict(status_dev=FAKE + MB), dict(out_dev=FAKE + 2 * MB), dict(out_dev=FAKE + 10 * MB), dict(token_dev=FAKE + 13 * MB)], ids=str)
def test_constraints_that_are_refused(bad):
    assert B.LIB.d3_constrain_logits(C.byref(logits_args(**bad)), None) == B.EINVAL


def test_constraints_without_rows_are_nothing_to_do():
    assert B.LIB.d3_constrain_logits(C.byref(logits_args(n_rows=0)), None) == B.OK


def refused(call, *args, **kw):
    with pytest.raises(B.D3Error) as e:
        call(*args, **kw)
    assert e.value.code == B.EINVAL


def test_the_binding_refuses():
    q = torch.zeros((300, 512), dtype=torch.float8_e4m3fn)
    s = torch.zeros((3, 4))
    for bad in (q[:, :504], q[:, ::2], q.view(torch.uint8), q[0]):
        refused(K.Weight8, bad, s)
    for bad in (s[:, :3], s.double(), torch.zeros((3, 8))[:, ::2], s[:2]):
        refused(K.Weight8, q, bad)
    w = K.Weight8(q, s)                                  # (host tensors make a handle, but no call)
    a, sc = torch.zeros((5, 512), dtype=torch.float8_e4m3fn), torch.zeros((5, 4))
    refused(K.d3_matmul8, a, sc, w)
    for args, kw in (((a[:, :256], sc), {}), ((a, sc[:, :3]), {}), ((a, sc.half()), {}), ((a.float(), sc), {}), ((a, sc), dict(out=torch.zeros((5, 299)))),
                     ((a, sc), dict(out=torch.zeros((4, 300)))), ((a, sc), dict(dtype=torch.float8_e4m3fn)), ((a, sc), dict(dtype=torch.float64)),
                     ((a, sc), dict(dtype=torch.float16, out=torch.zeros((5, 300)))), ((a, sc), dict(status=torch.zeros(1)))):
        refused(K.d3_matmul8, *args, w, **kw)
    refused(K.d3_gated_matmul8, a, sc, w, K.Weight8(q[:299], s))
    refused(K.d3_gated_matmul8, a, sc, w, w, dtype=torch.bfloat16, scale=torch.zeros((5, 3)))
    refused(K.d3_gated_matmul8, a, sc, w, w, scale=torch.zeros((5, 2)))
    x, g = torch.zeros((5, 256)), torch.zeros(256)
    for args, kw in (((x, g), {}), ((x[:, :12], g[:12]), {}), ((x.double(), g), {}), ((x, g[:8]), {}), ((x, g.double()), {}), ((x, g), dict(add=x.half())),
                     ((x, g), dict(add=x[:4])), ((x, g), dict(total=x)), ((x, g), dict(dtype=torch.int8)), ((x, g), dict(eps=-1.0)),
                     ((x, g), dict(dtype=torch.float32, scale=torch.zeros((5, 2)))), ((x, g), dict(scale=torch.zeros((5, 1)))),
                     ((x, g), dict(out=torch.zeros((5, 256)), dtype=torch.bfloat16)), ((x.t(), g), {})):
        refused(K.d3_add_norm, *args, **kw)
    refused(K.d3_quantize, x)
    refused(K.d3_quantize_weight, torch.zeros((8, 64)))
    z, h, one = torch.zeros((3, 1000)), torch.zeros((3, 20), dtype=torch.int32), torch.zeros(3)
    for kw in ({}, dict(history=h.long()), dict(history=h[:2]), dict(lengths=h[:, 0].contiguous()), dict(history=h, lengths=one), dict(history=h, repetition=one[:2]),
               dict(bias_ids=h), dict(bias=z[:, :20]), dict(bias_ids=h, bias=torch.zeros((3, 19))), dict(masks=torch.zeros((2, 32), dtype=torch.int32)),
               dict(masks=torch.zeros((2, 31), dtype=torch.int32), mask_of=h[:, 0].contiguous()), dict(out=torch.zeros((3, 999))), dict(token=one), dict(status=one)):
        refused(K.d3_constrain_logits, z, **kw)


def test_layouts_of_the_argument_structs():
    assert [C.sizeof(t) for t in (K.Weight8Args, K.AddNormArgs, K.Matmul8Args, K.ConstrainLogitsArgs)] == [48, 120, 88, 184]
