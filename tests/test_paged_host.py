"""Host side of the paged key-value operators (no GPU): what the C ABI and the binding refuse before
anything is enqueued, and the sizes they report."""
import ctypes as C

import pytest
import torch

from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import paged as P

FAKE = 1 << 20        # an aligned address that no refused call may touch


def kv_args(**kw):
    a = P.PagedKVArgs(C.sizeof(P.PagedKVArgs), P.BF16, 10, 16, 2, 64, 2 * 16 * 64, 16 * 64, 64, FAKE, FAKE, None, None, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def plan_args(**kw):
    a = P.PagePlanArgs(C.sizeof(P.PagePlanArgs), 3, 16, 10, 4, 8, 4, *[FAKE] * 11, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def append_args(**kw):
    a = P.PagedAppendArgs(C.sizeof(P.PagedAppendArgs), P.BF16, 5, 4, 100, FAKE, FAKE, 128, 64, 128, 64, FAKE, FAKE, 256, 64, 256, 64,
                          FAKE, FAKE, FAKE, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def attention_args(**kw):
    a = P.PagedAttentionArgs(C.sizeof(P.PagedAttentionArgs), P.BF16, 3, 4, 3, 8, 8, 0.125, FAKE, 256, 64, FAKE, 256, 64, None, FAKE,
                             FAKE, None, FAKE, 1 << 30, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_KV = [dict(struct_size=4), dict(dtype=P.FP32), dict(dtype=9), dict(n_pages=0), dict(page_size=8), dict(page_size=48),
          dict(page_size=2048), dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=256), dict(page_stride=0), dict(head_stride=63),
          dict(token_stride=68), dict(token_stride=-64), dict(k_dev=None), dict(v_dev=None), dict(k_dev=FAKE + 8), dict(v_dev=FAKE + 2),
          dict(k_scale_dev=FAKE)]


@pytest.mark.parametrize("bad", BAD_KV, ids=str)
def test_pools_that_are_refused(bad):
    kv = kv_args(**bad)
    assert B.LIB.d3_paged_append(C.byref(kv), C.byref(append_args()), None) == B.EINVAL
    assert B.LIB.d3_paged_attention(C.byref(kv), C.byref(attention_args()), None) == B.EINVAL


@pytest.mark.parametrize("bad", [
    dict(struct_size=0), dict(n_requests=0), dict(n_requests=4097), dict(page_size=17), dict(page_size=0), dict(n_pages=0),
    dict(table_width=0), dict(max_tokens=0), dict(table_stride=3), dict(table_width=1 << 27, table_stride=1 << 27),
    dict(cached_dev=None), dict(new_tokens_dev=None), dict(table_dev=None), dict(free_dev=None), dict(n_free_dev=None),
    dict(cached_out_dev=None), dict(n_free_out_dev=None), dict(first_dev=None), dict(slots_dev=None), dict(row_dev=None),
    dict(context_dev=None), dict(slots_dev=FAKE + 8), dict(row_dev=FAKE + 4), dict(context_dev=FAKE + 8), dict(table_dev=FAKE + 1),
    dict(status_dev=FAKE + 2)], ids=str)
def test_plans_that_are_refused(bad):
    assert B.LIB.d3_page_plan(C.byref(plan_args(**bad)), None) == B.EINVAL


@pytest.mark.parametrize("bad", [
    dict(struct_size=1), dict(dtype=P.FP16), dict(dtype=P.E4M3), dict(dtype=-1), dict(n_tokens=-1), dict(k_dev=None), dict(v_dev=None),
    dict(k_dev=FAKE + 4), dict(v_dev=FAKE + 8), dict(slots_dev=None), dict(slots_dev=FAKE + 4), dict(k_token_stride=-64),
    dict(k_head_stride=65), dict(v_token_stride=130), dict(v_head_stride=1 << 40), dict(rope_len=0), dict(rope_dev=FAKE + 8),
    dict(context_dev=None), dict(rope_dev=None), dict(n_q_heads=0), dict(q_out_dev=None), dict(q_dev=FAKE + 2), dict(q_out_dev=FAKE + 2),
    dict(q_token_stride=257), dict(q_out_token_stride=32), dict(q_out_head_stride=0), dict(status_dev=FAKE + 1),
    dict(n_q_heads=65536), dict(n_tokens=2 ** 31 - 1)], ids=str)
def test_appends_that_are_refused(bad):
    assert B.LIB.d3_paged_append(C.byref(kv_args()), C.byref(append_args(**bad)), None) == B.EINVAL


@pytest.mark.parametrize("bad", [
    dict(struct_size=1), dict(dtype=P.FP16), dict(dtype=P.E4M3), dict(n_rows=-1), dict(n_rows=65536, table_rows=70000), dict(n_q_heads=3),
    dict(n_q_heads=0), dict(table_rows=0), dict(table_rows=2), dict(table_width=0), dict(table_stride=7),
    dict(table_width=1 << 27, table_stride=1 << 27), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_dev=None),
    dict(q_dev=FAKE + 8), dict(q_row_stride=258), dict(q_head_stride=-64), dict(out_dev=None), dict(out_dev=FAKE + 1),
    dict(out_row_stride=32), dict(out_head_stride=0), dict(lse_dev=FAKE + 2), dict(table_dev=None), dict(context_dev=None),
    dict(rows_dev=FAKE + 1), dict(workspace_dev=None), dict(workspace_dev=FAKE + 128), dict(workspace_bytes=1000),
    dict(status_dev=FAKE + 2)], ids=str)
def test_attentions_that_are_refused(bad):
    assert B.LIB.d3_paged_attention(C.byref(kv_args()), C.byref(attention_args(**bad)), None) == B.EINVAL


def test_outputs_that_overlap_are_refused():
    for bad in (dict(q_out_token_stride=64), dict(q_out_head_stride=128), dict(q_out_token_stride=248)):
        assert B.LIB.d3_paged_append(C.byref(kv_args()), C.byref(append_args(**bad)), None) == B.EINVAL, bad
    for bad in (dict(head_stride=64), dict(page_stride=16 * 64), dict(page_stride=64), dict(token_stride=128)):
        kv = kv_args(**bad)
        assert B.LIB.d3_paged_append(C.byref(kv), C.byref(append_args()), None) == B.EINVAL, bad
        assert B.LIB.d3_paged_attention(C.byref(kv), C.byref(attention_args(n_rows=0)), None) == B.OK, bad    # reads alone
    for bad in (dict(out_row_stride=64), dict(out_head_stride=72), dict(out_row_stride=255)):
        assert B.LIB.d3_paged_attention(C.byref(kv_args()), C.byref(attention_args(**bad)), None) == B.EINVAL, bad
    nothing = dict(n_tokens=0)
    for kv in (kv_args(), kv_args(token_stride=128, head_stride=64, page_stride=2048), kv_args(page_stride=64, head_stride=640, token_stride=1280),
               kv_args(n_pages=1, page_stride=64)):
        assert B.LIB.d3_paged_append(C.byref(kv), C.byref(append_args(**nothing)), None) == B.OK
    for good in (dict(q_out_token_stride=64, q_out_head_stride=320), dict(q_out_token_stride=512, q_out_head_stride=128)):
        assert B.LIB.d3_paged_append(C.byref(kv_args()), C.byref(append_args(n_tokens=0, **good)), None) == B.OK


def test_null_arguments():
    n = C.c_size_t()
    assert B.LIB.d3_page_plan(None, None) == B.EINVAL
    assert B.LIB.d3_paged_append(None, None, None) == B.EINVAL and B.LIB.d3_paged_append(C.byref(kv_args()), None, None) == B.EINVAL
    assert B.LIB.d3_paged_attention(None, None, None) == B.EINVAL
    assert B.LIB.d3_paged_attention_workspace(None, 4, C.byref(n)) == B.EINVAL
    assert B.LIB.d3_paged_attention_workspace(C.byref(kv_args()), 4, None) == B.EINVAL
    assert B.LIB.d3_paged_attention_workspace(C.byref(kv_args()), 3, C.byref(n)) == B.EINVAL
    assert B.LIB.d3_paged_maps(None, FAKE) == B.EINVAL and B.LIB.d3_paged_maps(C.byref(kv_args()), None) == B.EINVAL
    assert B.LIB.d3_paged_maps(C.byref(kv_args()), FAKE + 32) == B.EINVAL
    assert B.LIB.d3_paged_view(None, 0, None, None, None, None) == B.EINVAL
    for bad in ((0, 64, 1e4, FAKE), (5, 48, 1e4, FAKE), (5, 64, 0.0, FAKE), (5, 64, float("nan"), FAKE), (5, 64, 1e4, None),
                (5, 64, 1e4, FAKE + 8), (2 ** 31 - 1, 128, 1e4, FAKE)):
        assert B.LIB.d3_rope_table(*bad, None) == B.EINVAL


def test_tensor_maps_of_another_pool_are_refused():
    kv, room = kv_args(), C.create_string_buffer(P.MAPS_BYTES + 64)
    kv.maps = (C.addressof(room) + 63) & ~63       # zeros: made for no pool
    assert B.LIB.d3_paged_attention(C.byref(kv), C.byref(attention_args(n_rows=0)), None) == B.EINVAL


def test_calls_without_work_return_at_once():
    assert B.LIB.d3_paged_append(C.byref(kv_args()), C.byref(append_args(n_tokens=0)), None) == B.OK
    assert B.LIB.d3_paged_attention(C.byref(kv_args()), C.byref(attention_args(n_rows=0)), None) == B.OK


def test_workspace_holds_two_pieces_per_multiprocessor():
    for dh in (32, 64, 128):
        n = C.c_size_t()
        assert B.LIB.d3_paged_attention_workspace(C.byref(kv_args(head_dim=dh, k_dev=None, v_dev=None)), 32, C.byref(n)) == B.OK
        assert n.value % 256 == 0 and n.value >= 2 * 148 * 16 * (dh + 2) * 4


def test_struct_sizes_match_the_header():
    assert [C.sizeof(t) for t in (P.PagedKVArgs, P.PagePlanArgs, P.PagedAppendArgs, P.PagedAttentionArgs)] == [88, 128, 152, 144]


def pool(**kw):
    shape = dict(n=6, h=2, p=16, d=64, dtype=torch.bfloat16)
    shape.update(kw)
    return torch.zeros((shape["n"], shape["h"], shape["p"], shape["d"]), dtype=shape["dtype"])


def refused(f, *args, **kw):
    with pytest.raises(B.D3Error) as e:
        f(*args, **kw)
    assert e.value.code == B.EINVAL


def test_binding_refusals():
    cache = P.PagedKV(pool(), pool())
    refused(P.PagedKV, pool(), pool(p=32))
    refused(P.PagedKV, pool(), pool(dtype=torch.float16))
    refused(P.PagedKV, pool(dtype=torch.float32), pool(dtype=torch.float32))
    refused(P.PagedKV, pool(d=96), pool(d=96))
    refused(P.PagedKV, pool(p=24), pool(p=24))
    refused(P.PagedKV, pool().transpose(2, 3), pool().transpose(2, 3))
    refused(P.PagedKV, pool(), pool().permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))
    refused(P.PagedKV, pool(), pool(), torch.ones(2), torch.ones(2))
    e4 = dict(dtype=torch.float8_e4m3fn)
    P.PagedKV(pool(**e4), pool(**e4), torch.ones(2), None)
    refused(P.PagedKV, pool(**e4), pool(**e4), torch.ones(3), None)
    q, ctx, table = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32)
    refused(P.d3_paged_attention, cache, q, table, ctx)                        # not on a CUDA device
    refused(P.d3_paged_attention, cache, q[0], table, ctx)
    refused(P.d3_paged_attention, cache, q[..., :32], table, ctx)
    refused(P.d3_paged_attention, cache, q, table.long(), ctx)
    refused(P.d3_paged_attention, cache, q, table, ctx[:2])
    refused(P.d3_paged_attention, cache, q, table, ctx, rows=ctx[:2])
    refused(P.d3_paged_attention, cache, q, table, ctx, out=q[:2])
    refused(P.d3_paged_attention, cache, q, table, ctx, lse=torch.zeros(3, 5))
    refused(P.d3_paged_attention, cache, q, table, ctx, workspace=torch.zeros(5, 2)[:, 0])
    x, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    rope = torch.zeros(7, 32, 2)
    refused(P.d3_paged_append, cache, x, x, slots)                             # not on a CUDA device
    refused(P.d3_paged_append, cache, x, x[:2], slots)
    refused(P.d3_paged_append, cache, x, x, slots.int())
    refused(P.d3_paged_append, cache, x, x.float(), slots)
    refused(P.d3_paged_append, cache, x, x, slots, rope=rope)
    refused(P.d3_paged_append, cache, x, x, slots, rope=rope[..., :1], context=ctx)
    refused(P.d3_paged_append, cache, x, x, slots, q=q)
    refused(P.d3_paged_append, cache, x, x, slots, q_out=q)
    refused(P.d3_paged_append, cache, x, x, slots, q=q, q_out=q.float(), rope=rope, context=ctx)
    refused(P.d3_paged_append, cache, x, x, slots, status=ctx)
    free, one = torch.zeros(9, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    good = dict(cached=ctx, new_tokens=ctx.clone(), table=table, free=free, n_free=one, page_size=16, max_tokens=4)
    refused(P.PagePlan(**good).d3_page_plan)                                   # not on a CUDA device
    for bad in (dict(table=table[:2]), dict(table=table.long()), dict(new_tokens=ctx[:2]), dict(n_free=free), dict(max_tokens=0),
                dict(cached=ctx.long()), dict(cached_out=ctx[:2]), dict(status=free), dict(free=free[None])):
        refused(P.PagePlan, **{**good, **bad})
    refused(P.d3_rope_table, 5, 48, device="cpu")
    refused(P.d3_rope_table, 5, 64, device="cpu")


def test_strides_of_single_entries_do_not_matter():
    one = torch.zeros(64, dtype=torch.bfloat16).as_strided((1, 1, 64), (3, 5, 1))
    assert P._strides(one) == [64, 64]
    assert P._strides(torch.zeros(2, 5, 64)[:, 1:2]) == [320, 64]
    P.PagedKV(torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16).as_strided((1, 1, 16, 64), (1, 1, 64, 1)),
              torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16))
