"""Paged key-value operators (plan, append, attention) against plain 64-bit forms.

Tolerances.  A result stored in t bits is off by at most half a step: eps(t) / 2 of its value.  Before
that rounding the attention kernel works in fp32, so with A = sum_t p_t |v_t| / sum_t p_t its result is
off by at most E * A, where E adds up
  2 d     d = the largest error of a score: (dh + 8) fp32 roundings of at most scale * sum |q_d k_d|
          (a weight is off by a factor e^d, numerator and denominator both)
  2^-16   what is left of a weight after its two bf16 terms (2^-8 of it after the first, 2^-8 of that after the second);
          2^-21 with two fp16 or three bf16 ones (2^-22, 2^-24); 2^-10 with one fp16 term (8-bit cache, bf16 result:
          2^-11 of it, and as much again for sums that use the unrounded weights)
  c 2^-23 c = sums of length/16 tensor-core steps and the joining of warps and CTAs
  2^-20   two exponentials of 2^-22 each (the weight, the rescaling) in numerator and denominator
The rotary products and sums of append are rounded one by one, so its results are compared bit for bit
with the same fp32 operations in torch, and to half a step with 64-bit ones.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def paged():
    from paper_2503_08524_b200 import paged as P
    return P


def pool(n_pages, hkv, page, dh, dtype, layout="head", seed=0, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    shape = (n_pages, hkv, page, dh) if layout == "head" else (n_pages, page, hkv, dh)
    kv = []
    for _ in range(2):
        x = torch.empty(shape, dtype=FP16 if dtype == E4M3 else dtype, device=DEV).normal_(0.0, std, generator=g)
        x = x.to(dtype)
        kv.append(x if layout == "head" else x.permute(0, 2, 1, 3))
    return kv


def tables(contexts, page, n_pages, seed, spare=1, fill=-1):
    """Disjoint pages for the rows, in random order; entries behind them `fill`."""
    counts = [-(-c // page) for c in contexts]
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(counts + [1]) + spare
    t = torch.full((len(contexts), width), fill, dtype=torch.int32)
    for b, n in enumerate(counts):
        t[b, :n] = torch.tensor(order[:n], dtype=torch.int32)
        order = order[n:]
    return t.to(DEV)


def dense(cache, pages, n):
    """[kv head][n][dim] in 64 bits."""
    x = torch.stack([cache[p].to(FP32) for p in pages]) if pages else cache[:0].to(FP32)
    return x.double().permute(1, 0, 2, 3).reshape(cache.shape[1], -1, cache.shape[3])[:, :n]


def reference(q, k, v, scale, terms_eps):
    """(out, lse, allowed error before the last rounding) of one row; q [hq][dh], k, v [hkv][n][dh], fp64."""
    hq, dh = q.shape
    hkv, n = k.shape[:2]
    qg = q.reshape(hkv, hq // hkv, dh)
    s = qg @ k.transpose(1, 2) * scale
    p = torch.softmax(s, -1)
    out, A = p @ v, p @ v.abs()
    d = (dh + 8) * 2.0 ** -23 * abs(scale) * (qg.abs() @ k.abs().transpose(1, 2)).amax(-1, keepdim=True)
    E = 2 * d + terms_eps + (n / 16 + 200) * 2.0 ** -23 + 2.0 ** -20
    lse = torch.logsumexp(s, -1)
    return out.reshape(hq, dh), lse.reshape(hq), (E * A).reshape(hq, dh), (E.squeeze(-1) + lse.abs() * 2.0 ** -22).reshape(hq)


def check(out, lse, q, cache, table, contexts, scale=None, rows=None):
    k, v = cache.k, cache.v
    dh, page = k.shape[3], k.shape[2]
    scale = dh ** -0.5 if scale is None else scale
    half = torch.finfo(out.dtype).eps / 2
    t = table.cpu().tolist()
    terms = 2.0 ** -16 if k.dtype == BF16 and q.dtype == BF16 else 2.0 ** -10 if k.dtype == E4M3 and q.dtype == BF16 else 2.0 ** -21
    for b, n in enumerate(contexts):
        r = b if rows is None else rows[b]
        if r < 0:
            continue
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all(), b
            continue
        pages = t[r][: -(-n // page)]
        kd, vd = dense(k, pages, n), dense(v, pages, n)
        if cache.k_scale is not None:
            kd = kd * cache.k_scale.double()[:, None, None]
        if cache.v_scale is not None:
            vd = vd * cache.v_scale.double()[:, None, None]
        want, want_lse, tol, tol_lse = reference(q[b].double(), kd, vd, scale, terms)
        err = (out[b].double() - want).abs()
        allowed = half * (want.abs() + tol) + tol + torch.finfo(out.dtype).smallest_normal * half * 2
        assert (err <= allowed).all(), (b, n, float((err / allowed).max()))
        assert ((lse[b].double() - want_lse).abs() <= tol_lse).all(), (b, n)


def make(paged, contexts, hq, hkv, dh, page, kv, x, layout="head", seed=0, scales=None, q_std=1.5):
    n_pages = sum(-(-c // page) for c in contexts) + 2
    k, v = pool(n_pages, hkv, page, dh, kv, layout, seed, 30.0 if kv == E4M3 else 1.0)
    ks = vs = None
    if kv == E4M3 and scales != "none":
        ks = torch.linspace(0.02, 0.05, hkv, device=DEV)
        vs = torch.linspace(0.06, 0.03, hkv, device=DEV)
    cache = paged.PagedKV(k, v, ks, vs)
    table = tables(contexts, page, n_pages, seed + 1)
    q = torch.empty((len(contexts), hq, dh), dtype=x, device=DEV).normal_(0.0, q_std, generator=torch.Generator(DEV).manual_seed(seed + 2))
    return cache, table, q, torch.tensor(contexts, dtype=torch.int32, device=DEV)


def poison_behind(cache, table, contexts):
    """NaN in every position of the rows' last pages behind their context, and in every page no row has."""
    page = cache.page_size
    used = set()
    for b, n in enumerate(contexts):
        ids = table[b].tolist()[: -(-n // page)]
        used |= set(ids)
        if n % page:
            for t in (cache.k, cache.v):
                t[ids[-1], :, n % page:, :] = torch.tensor(math.nan, device=DEV).to(t.dtype)
    rest = [p for p in range(cache.n_pages) if p not in used]
    for t in (cache.k, cache.v):
        for p in rest:
            t[p] = torch.full((), math.nan, device=DEV).to(t.dtype)


LENGTHS = [1, 2, 15, 16, 17, 31, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 500, 0]


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (FP16, FP16), (E4M3, BF16), (E4M3, FP16)],
                         ids=["bf16", "bf16-fp32", "fp16", "e4m3-bf16", "e4m3-fp16"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (16, 2), (16, 1), (7, 7), (48, 3), (5, 1), (18, 1), (40, 2)])
def test_attention_types_heads_and_lengths(paged, kv, x, dh, hq, hkv):
    page, layout = (16, "head") if (hq + dh // 32) % 2 else (64, "token")
    cache, table, q, ctx = make(paged, LENGTHS, hq, hkv, dh, page, kv, x, layout, seed=hq * 100 + dh)
    poison_behind(cache, table, LENGTHS)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True, status=status)
    assert int(status) == 0
    check(out, lse, q, cache, table, LENGTHS)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_attention_page_sizes_and_long_rows(paged, page, layout):
    contexts = [5000, 1, 3001, 64, 1023, 1025, 12345]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 128, page, BF16, BF16, layout, seed=page)
    poison_behind(cache, table, contexts)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
    check(out, lse, q, cache, table, contexts)


@pytest.mark.parametrize("n,hq,hkv", [(1, 8, 1), (1, 32, 32), (3, 64, 8), (700, 4, 4), (1100, 2, 1), (128, 3, 3), (129, 3, 3)])
def test_attention_row_counts(paged, n, hq, hkv):
    """One row cut over all SMs; more rows than threads of a CTA."""
    contexts = [40000] if n == 1 and hkv == 1 else [777, 1500, 2048][:n] if n <= 3 else [(37 * i) % 130 for i in range(n)]
    cache, table, q, ctx = make(paged, contexts, hq, hkv, 64, 32, FP16, FP16, seed=n)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
    check(out, lse, q, cache, table, contexts)


@pytest.mark.parametrize("contexts", [[2000] * 4, [1100] * 9, [700, 640, 0, 655], [3000, 1, 1, 1, 1, 1], [500] * 40], ids=str)
def test_attention_whole_and_cut_rows(paged, contexts):
    """Rows of like lengths stay whole in one CTA, others are cut: the results do not tell."""
    cache, table, q, ctx = make(paged, contexts, 32, 32, 128, 64, BF16, BF16, seed=len(contexts))
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
    check(out, lse, q, cache, table, contexts)
    wide = torch.full((len(contexts), 4000), -1, dtype=torch.int32, device=DEV)      # room for more than any row has
    wide[:, :table.shape[1]] = table
    out, lse = paged.d3_paged_attention(cache, q, wide, ctx, with_lse=True)
    check(out, lse, q, cache, table, contexts)


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (FP16, FP16), (E4M3, BF16), (E4M3, FP16)],
                         ids=["bf16", "bf16-fp32", "fp16", "e4m3-bf16", "e4m3-fp16"])
@pytest.mark.parametrize("dh,page", [(32, 256), (64, 16), (128, 64)])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (5, 1), (12, 1), (19, 1)])
def test_attention_few_rows_of_wide_tables(paged, kv, x, dh, page, hq, hkv):
    """Clusters of CTAs share a row: more pieces than units, fewer, none; padding rows; a row that ends in a unit's first tile."""
    contexts = [1700, 1, 0, 65, 257, 1024]
    cache, table, q, ctx = make(paged, contexts, hq, hkv, dh, page, kv, x, seed=hq + dh)
    poison_behind(cache, table, contexts)
    rows = [0, 1, 2, 3, -1, 5]
    out, lse = torch.full_like(q, 7.0), torch.full((6, hq), 5.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for _ in range(3):
        paged.d3_paged_attention(cache, q, table, ctx, rows=torch.tensor(rows, dtype=torch.int32, device=DEV), out=out, lse=lse,
                                 status=status)
    assert int(status) == 0 and (out[4] == 7.0).all() and (lse[4] == 5.0).all()
    check(out, lse, q, cache, table, contexts, rows=rows)


def test_attention_few_rows_of_wide_tables_with_bad_device_data(paged):
    contexts = [1000, 700, 90]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 128, 16, BF16, BF16, seed=26)
    ids = table[0].tolist()[:63]
    for bad in (-1, cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[0, 3], t[0, 62], t[0, 20:40] = bad, bad, bad       # a page, the last one, whole units of several CTAs
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = paged.d3_paged_attention(cache, q, t, ctx, with_lse=True, status=status)
        assert int(status) == -1
        kd, vd = dense(cache.k, ids, 1000), dense(cache.v, ids, 1000)
        keep = [i for i in range(992) if i // 16 != 3 and not 20 <= i // 16 < 40]
        want, want_lse, tol, tol_lse = reference(q[0].double(), kd[:, keep], vd[:, keep], 128 ** -0.5, 2.0 ** -16)
        assert ((out[0].double() - want).abs() <= 2.0 ** -8 * (want.abs() + tol) + tol).all()
        assert ((lse[0].double() - want_lse).abs() <= tol_lse).all()
        check(out[1:], lse[1:], q[1:], cache, table[1:], contexts[1:])
    t = torch.full_like(table, -5)                             # no page at all
    out, lse = paged.d3_paged_attention(cache, q, t, ctx, with_lse=True, status=status)
    assert (out == 0).all() and (lse == -math.inf).all()
    for bad in (-1, 16 * table.shape[1] + 1, 2 ** 31 - 1):
        status.zero_()
        c = ctx.clone()
        c[1] = bad
        out, lse = paged.d3_paged_attention(cache, q, table, c, with_lse=True, status=status)
        assert int(status) == -1
        check(out, lse, q, cache, table, [1000, 0, 90])
    status.zero_()
    out = torch.full_like(q, 3.0)
    rows = torch.tensor([0, 3, -7], dtype=torch.int32, device=DEV)
    paged.d3_paged_attention(cache, q, table, ctx, rows=rows, out=out, status=status)
    assert int(status) == -1 and (out[1:] == 3.0).all() and not (out[0] == 3.0).all()


def test_attention_few_rows_captured_and_replayed_with_other_lengths(paged):
    contexts = [1500, 1500, 1500]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 128, 16, BF16, BF16, seed=31)
    ws, out, lse = paged.attention_workspace(cache, 8), torch.zeros_like(q), torch.zeros((3, 8), device=DEV)
    call = lambda: paged.d3_paged_attention(cache, q, table, ctx, out=out, lse=lse, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for lengths in ([1500, 1, 0], [64, 65, 1499], [0, 0, 0], [1, 1, 1], [1024, 1500, 700]):
        ctx.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        check(out, lse, q, cache, table, lengths)
        bits = out.clone()
        call()
        assert torch.equal(out, bits)


FIRST_CALL = """
import torch
from paper_2503_08524_b200 import paged as P
dev = "cuda:0"
k, v = (torch.randn(40, 2, 16, 64, device=dev).bfloat16() for _ in range(2))
cache = P.PagedKV(k, v)
q, new = torch.randn(2, 8, 64, device=dev).bfloat16(), torch.randn(2, 2, 64, device=dev).bfloat16()
i32 = dict(dtype=torch.int32, device=dev)
table = torch.arange(40, **i32).view(2, 20)
n_free = torch.zeros(1, **i32)
plan = P.PagePlan(cached=torch.tensor([99, 300], **i32), new_tokens=torch.tensor([1, 1], **i32), table=table, free=torch.zeros(40, **i32),
                  n_free=n_free, page_size=16, max_tokens=2, cached_out=torch.zeros(2, **i32), n_free_out=torch.zeros(1, **i32))
rope = P.d3_rope_table(400, 64)
q_out, out, ws = torch.zeros_like(q), torch.zeros_like(q), P.attention_workspace(cache, 8)
def step():
    plan.d3_page_plan()
    P.d3_paged_append(cache, new, new, plan.slots, q=q, q_out=q_out, rope=rope, context=plan.context)
    P.d3_paged_attention(cache, q_out, table, plan.context, rows=plan.row, out=out, workspace=ws)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
assert not out.any()
graph.replay()
got = out.clone()
step()
assert int(plan.status) == 0 and got.any() and torch.equal(out, got), (got, out)
"""


def test_the_first_calls_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (E4M3, BF16)], ids=["bf16", "bf16-fp32", "e4m3-bf16"])
@pytest.mark.parametrize("dh,hq,hkv", [(128, 16, 2), (64, 6, 2), (32, 32, 2), (128, 3, 3)])
@pytest.mark.parametrize("long", [0, 3000])
def test_attention_many_short_rows(paged, kv, x, dh, hq, hkv, long):
    """Many row ends close together, lengths 0 to 300, alone (no row is cut) and beside a long row (rows are cut); equal bits each time."""
    g = torch.Generator().manual_seed(dh + hq + long)
    contexts = torch.randint(0, 301, (260,), generator=g).tolist()
    contexts[7:40] = [n % 17 for n in contexts[7:40]]
    if long:
        contexts[100] = long
    cache, table, q, ctx = make(paged, contexts, hq, hkv, dh, 16, kv, x, seed=41)
    first = None
    for _ in range(4):
        out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
        if first is None:
            first = (out, lse)
            check(out, lse, q, cache, table, contexts)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_attention_peaked_scores_and_far_tails(paged):
    """One position outweighs the rest by e^16, in every type: the tail still counts (fp16 weights of 2^-24 and below)."""
    for kv, x in ((BF16, BF16), (FP16, FP16), (E4M3, FP16), (BF16, FP32)):
        n, dh = 4000, 64
        cache, table, q, ctx = make(paged, [n], 4, 1, dh, 64, kv, x, seed=9, scales="none")
        one = 0.25 if kv == E4M3 else 1.0
        cache.k.zero_()
        q.zero_()
        q[:, :, 0] = 16.0 / one * 8.0      # times 2^-3 (scale), times `one` = 16
        ids = table[0].tolist()
        cache.k[ids[3], 0, 5, 0] = one
        cache.v.copy_((cache.v.float().abs() * (0.1 if kv == E4M3 else 1.0)).to(kv))
        cache.v[ids[3], 0, 5] = 0.0
        out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
        check(out, lse, q, cache, table, [n])


def test_attention_large_queries_over_an_8_bit_cache(paged):
    """bf16 queries beyond fp16's range, and tiny ones: the power of two taken out of them comes back."""
    for mag in (1e6, 1e-30, 1e30):
        cache, table, q, ctx = make(paged, [200, 33], 8, 2, 64, 16, E4M3, BF16, seed=3, scales="none")
        q.copy_((q.float().clamp(-1, 1) * mag).to(BF16))
        scale = 0.01 / mag
        out, lse = paged.d3_paged_attention(cache, q, table, ctx, scale=scale, with_lse=True)
        check(out, lse, q, cache, table, [200, 33], scale=scale)


def test_attention_rows_map_padding_and_strided_tensors(paged):
    contexts = [300, 0, 45, 64, 129]
    cache, table, _, _ = make(paged, contexts, 8, 4, 64, 16, BF16, BF16, seed=4)
    rows = [4, -1, 0, 2, -1, 1, 0]
    n = len(rows)
    ctx = [contexts[r] if r >= 0 else 99999999 for r in rows]
    ctx[6] = 17                                     # a second row over the same pages, cut short
    big = torch.empty((n, 20, 80), dtype=BF16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(5))
    q = big[:, 3:11, 8:72]                          # strides 1600, 80, offset 16-byte aligned
    out_big = torch.full((n, 9, 71), 7.0, dtype=BF16, device=DEV)
    out = out_big[:, :8, 3:67]
    lse = torch.full((n, 8), 5.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = paged.d3_paged_attention(cache, q, table, torch.tensor(ctx, dtype=torch.int32, device=DEV), out=out, lse=lse,
                                   rows=torch.tensor(rows, dtype=torch.int32, device=DEV), status=status)
    assert got[0] is out and got[1] is lse and int(status) == 0
    check(out, lse, q, cache, table, ctx, rows=rows)
    for b in (1, 4):                                # padding rows as they were
        assert (out[b] == 7.0).all() and (lse[b] == 5.0).all()
    out_big[:, :8, 3:67] = 7.0
    assert (out_big == 7.0).all()                   # nothing written beside `out`


def test_attention_takes_a_table_of_one_unit_and_tables_of_one_row(paged):
    for contexts in ([64], [7, 64, 0, 16]):
        cache, table, q, ctx = make(paged, contexts, 4, 4, 32, 64, BF16, BF16, seed=8)
        t = table[:, :1].contiguous()
        out, lse = paged.d3_paged_attention(cache, q, t, ctx, with_lse=True)
        check(out, lse, q, cache, t, contexts)


def test_attention_bad_device_data_is_reported_and_left_out(paged):
    contexts = [200, 100, 90]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 64, 16, BF16, BF16, seed=6)
    for bad in (-1, cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[0, 3] = bad                               # positions 48..63 of row 0 are left out
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = paged.d3_paged_attention(cache, q, t, ctx, with_lse=True, status=status)
        assert int(status) == -1
        ids = table[0].tolist()[:13]
        kd, vd = dense(cache.k, ids, 200), dense(cache.v, ids, 200)
        keep = [i for i in range(200) if not 48 <= i < 64]
        want, want_lse, tol, tol_lse = reference(q[0].double(), kd[:, keep], vd[:, keep], 64 ** -0.5, 2.0 ** -16)
        assert ((out[0].double() - want).abs() <= 2.0 ** -8 * (want.abs() + tol) + tol).all()
        assert ((lse[0].double() - want_lse).abs() <= tol_lse).all()
        check(out[1:], lse[1:], q[1:], cache, table[1:], contexts[1:])
    for bad in (-1, 16 * table.shape[1] + 1, 2 ** 31 - 1):
        status.zero_()
        c = ctx.clone()
        c[1] = bad
        out, lse = paged.d3_paged_attention(cache, q, table, c, with_lse=True, status=status)
        assert int(status) == -1 and (out[1] == 0).all() and (lse[1] == -math.inf).all()
        check(out, lse, q, cache, table, [200, 0, 90])
    status.zero_()
    out = torch.full_like(q, 3.0)
    rows = torch.tensor([0, 3, -7], dtype=torch.int32, device=DEV)
    paged.d3_paged_attention(cache, q, table, ctx, rows=rows, out=out, status=status)
    assert int(status) == -1 and (out[1:] == 3.0).all() and not (out[0] == 3.0).all()


def test_attention_nan_inside_the_context_shows(paged):
    cache, table, q, ctx = make(paged, [100, 100], 4, 4, 64, 16, BF16, BF16, seed=7)
    cache.k[int(table[0, 2]), 1, 3, 5] = math.nan
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
    assert out[0, 1].isnan().all() and lse[0, 1].isnan()
    assert not out[0, [0, 2, 3]].isnan().any() and not out[1].isnan().any()


def test_attention_equal_inputs_give_equal_bits_and_ignore_the_workspace(paged):
    contexts = [4097, 3, 900, 0, 2500]
    cache, table, q, ctx = make(paged, contexts, 16, 4, 128, 32, BF16, BF16, seed=11)
    ws = paged.attention_workspace(cache, 16)
    first = None
    for fill in (0, 255, 85):
        ws.fill_(fill)
        out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True, workspace=ws)
        if first is None:
            first = (out.clone(), lse.clone())
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_attention_with_and_without_the_pools_maps(paged):
    cache, table, q, ctx = make(paged, [300, 5], 8, 2, 64, 32, BF16, BF16, seed=13)
    want = paged.d3_paged_attention(cache, q, table, ctx)
    maps, cache.args.maps = cache.args.maps, None
    assert torch.equal(paged.d3_paged_attention(cache, q, table, ctx), want)
    cache.args.maps, cache.args.n_pages = maps, cache.n_pages - 1
    with pytest.raises(paged.D3Error):
        paged.d3_paged_attention(cache, q, table, ctx)


def test_attention_entries_beyond_32_bit_offsets(paged):
    """A pool of more than 2^32 bytes and 2^31 elements per tensor; the row's pages sit at its two ends."""
    hkv, page, dh = 8, 64, 128
    n_pages = (1 << 31) // (hkv * page * dh) + 40
    k = torch.empty((n_pages, hkv, page, dh), dtype=BF16, device=DEV)
    v = torch.empty_like(k)
    cache = paged.PagedKV(k, v)
    ids = [n_pages - 1, 0, n_pages - 2, 1, n_pages - 3]
    n = 4 * page + 9
    g = torch.Generator(DEV).manual_seed(1)
    kx, vx, q = (torch.empty((n if i < 2 else 1, hkv, dh), dtype=BF16, device=DEV).normal_(generator=g) for i in range(3))
    table = torch.tensor([ids], dtype=torch.int32, device=DEV)
    slots = torch.tensor([ids[i // page] * page + i % page for i in range(n)], device=DEV)
    paged.d3_paged_append(cache, kx, vx, slots)
    out, lse = paged.d3_paged_attention(cache, q, table, torch.tensor([n], dtype=torch.int32, device=DEV), with_lse=True)
    want, want_lse, tol, tol_lse = reference(q[0].double(), kx.double().transpose(0, 1), vx.double().transpose(0, 1), dh ** -0.5, 2.0 ** -16)
    assert ((out[0].double() - want).abs() <= 2.0 ** -8 * (want.abs() + tol) + tol).all()
    assert ((lse[0].double() - want_lse).abs() <= tol_lse).all()


# ---------------------------------------------------------------------------------------------- append
def rotated(x, rope, context):
    cs = rope[context.long() - 1][:, None]
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)


def stored(x, scale, dtype):
    if dtype == E4M3:
        if scale is not None:
            x = x / scale[:, None]
        x = x.clamp(-448.0, 448.0)
    return x.to(dtype)


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (FP16, FP16), (E4M3, BF16), (E4M3, FP16)],
                         ids=["bf16", "bf16-fp32", "fp16", "e4m3-bf16", "e4m3-fp16"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("n,hq,hkv,layout", [(1, 4, 4, "head"), (33, 7, 7, "token"), (3001, 64, 8, "head"), (20000, 3, 1, "token")])
def test_append_types_sizes_and_layouts(paged, kv, x, dh, n, hq, hkv, layout):
    page = 32
    n_pages = n // page + 5
    g = torch.Generator(DEV).manual_seed(n + dh)
    k, v = pool(n_pages, hkv, page, dh, kv, layout, seed=n)
    sc = (torch.linspace(0.01, 0.3, hkv, device=DEV), torch.linspace(0.4, 0.02, hkv, device=DEV)) if kv == E4M3 else (None, None)
    cache = paged.PagedKV(k, v, *sc)
    qkv = torch.empty((n, hq + 2 * hkv, dh), dtype=x, device=DEV).normal_(0.0, 3.0, generator=g)
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(n))[:n].to(DEV)
    slots[::5] = -1 if n > 1 else slots[::5]
    context = torch.randint(1, 4000, (n,), generator=g, device=DEV, dtype=torch.int32)
    context[slots < 0] = 0
    rope = paged.d3_rope_table(4000, dh)
    pos = torch.arange(4000, device=DEV, dtype=torch.float64)
    angle = pos[:, None] * 10000.0 ** (-2.0 * torch.arange(dh // 2, device=DEV, dtype=torch.float64) / dh)
    assert ((rope.double() - torch.stack([angle.cos(), angle.sin()], -1)).abs() <= 2.0 ** -24).all()
    before_k, before_v = k.clone(), v.clone()
    q, kx, vx = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    q_out = torch.full((n, hq, dh), 9.0, dtype=x, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    paged.d3_paged_append(cache, kx, vx, slots, q=q, q_out=q_out, rope=rope, context=context, status=status)
    assert int(status) == 0
    live = slots >= 0
    want_k, want_v = before_k.clone(), before_v.clone()
    for want, new, s in ((want_k, rotated(kx[live], rope, context[live]), sc[0]), (want_v, vx[live].float(), sc[1])):
        bits = torch.uint8 if kv == E4M3 else torch.int16
        want.view(bits).permute(0, 2, 1, 3)[slots[live] // page, slots[live] % page] = stored(new, s, kv).view(bits)
    bits = torch.uint8 if kv == E4M3 else torch.int16
    assert torch.equal(k.view(bits), want_k.view(bits)) and torch.equal(v.view(bits), want_v.view(bits))
    q64 = torch.full((n, hq, dh), 9.0, dtype=torch.float64, device=DEV)
    cs = rope.double()[context[live].long() - 1][:, None]
    a, b = q[live].double().chunk(2, -1)
    q64[live] = torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)
    reach = (a.abs() + b.abs()).repeat(1, 1, 2)
    assert torch.equal(q_out[live], rotated(q[live], rope, context[live]).to(x)) and (q_out[~live] == 9.0).all()
    err = (q_out[live].double() - q64[live]).abs()
    fp32_part = 3 * 2.0 ** -24 * reach          # two products and a sum, half a step each
    # below the smallest normal number a step is smallest_normal * eps whatever the value
    floor = torch.finfo(x).smallest_normal * torch.finfo(x).eps / 2
    assert (err <= torch.finfo(x).eps / 2 * (q64[live].abs() + fp32_part) + fp32_part + floor).all()
    paged.d3_paged_append(cache, kx, vx, slots, q=q, q_out=q, rope=rope, context=context)      # in place
    assert torch.equal(q[live], q_out[live])


def test_append_without_rotation_saturates_and_keeps_nan(paged):
    k, v = pool(3, 1, 16, 32, E4M3)
    cache = paged.PagedKV(k, v)
    x = torch.zeros((2, 1, 32), dtype=FP16, device=DEV)
    x[0, 0, :6] = torch.tensor([500.0, -60000.0, math.inf, -math.inf, math.nan, 0.001], dtype=FP16)
    x[1, 0, :4] = torch.tensor([448.0, 464.0, 17.0, 19.0], dtype=FP16)   # 17, 19: ties between 16, 18, 20
    paged.d3_paged_append(cache, x, x, torch.tensor([17, 40], device=DEV))
    a, b = k[1, 0, 1].float(), v[2, 0, 8].float()
    assert a[:4].tolist() == [448.0, -448.0, 448.0, -448.0] and a[4].isnan() and float(a[5]) == 2.0 ** -9 * round(0.001 * 512)
    assert b[:4].tolist() == [448.0, 448.0, 16.0, 20.0]


@pytest.mark.parametrize("scale", [1.0, 3e-3, 1e-25, 1e25, 2.0 ** -130, float("inf"), -0.7])
def test_append_division_by_any_scale(paged, scale):
    """What is stored is x / scale, rounded once to fp32 and then to 8 bits, for ordinary and for extreme numbers."""
    g = torch.Generator(DEV).manual_seed(4)
    n, dh = 4096, 64
    x = torch.empty((n, 1, dh), dtype=BF16, device=DEV).normal_(generator=g)
    x = (x.float() * 10.0 ** torch.empty((n, 1, 1), device=DEV).uniform_(-30, 30, generator=g)).to(BF16)
    x[0, 0, :8] = torch.tensor([0.0, -0.0, math.inf, -math.inf, 1e38, -1e38, 1e-38, 3e-39])
    k, v = pool(n // 16, 1, 16, dh, E4M3)
    sc = torch.full((1,), scale, device=DEV)
    paged.d3_paged_append(paged.PagedKV(k, v, sc, sc), x, x, torch.arange(n, device=DEV))
    want = (x.float() / sc).clamp(-448.0, 448.0).to(E4M3).float().reshape(n, dh)
    for t in (k, v):
        got = t.float().permute(0, 2, 1, 3).reshape(n, dh)
        assert torch.equal(got.nan_to_num(9e9), want.nan_to_num(9e9))


def test_append_a_rotary_table_beyond_the_unit_circle(paged):
    """Tables that also scale (or hold anything else) are taken as they are."""
    x = torch.full((16, 1, 64), 3e4, dtype=FP16, device=DEV)
    k, v = pool(1, 1, 16, 64, E4M3)
    one = torch.ones(1, device=DEV)
    rope = torch.tensor([[1e35, -1e35], [2.0, 0.5], [1e-3, 1e-3]], device=DEV)[:, None, :].expand(3, 32, 2).contiguous()
    ctx = torch.tensor([1 + i % 3 for i in range(16)], dtype=torch.int32, device=DEV)
    paged.d3_paged_append(paged.PagedKV(k, v, one, one), x, x, torch.arange(16, device=DEV), rope=rope, context=ctx)
    want = rotated(x, rope, ctx).clamp(-448.0, 448.0).to(E4M3).float()      # (inf - inf among it)
    assert torch.equal(k.float().permute(0, 2, 1, 3).reshape(16, 1, 64).nan_to_num(9e9), want.nan_to_num(9e9))


def test_append_bad_slots_and_positions_are_skipped_and_reported(paged):
    k, v = pool(4, 2, 16, 64, BF16)
    cache = paged.PagedKV(k, v)
    x = torch.ones((3, 2, 64), dtype=BF16, device=DEV)
    rope = paged.d3_rope_table(10, 64)
    for slots, ctx in (([5, 64, 7], [1, 1, 1]), ([5, 2 ** 40, 7], [1, 1, 1]), ([5, 6, 7], [1, 11, 1]), ([5, 6, 7], [1, 0, 1])):
        k.zero_(), v.zero_()
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        paged.d3_paged_append(cache, x, x, torch.tensor(slots, device=DEV), rope=rope,
                              context=torch.tensor(ctx, dtype=torch.int32, device=DEV), status=status)
        assert int(status) == -1
        assert (v[0, :, [5, 7]] == 1).all() and int((v != 0).sum()) == 2 * 2 * 64


def test_append_nothing(paged):
    k, v = pool(2, 2, 16, 64, BF16)
    x = torch.empty((0, 2, 64), dtype=BF16, device=DEV)
    assert paged.d3_paged_append(paged.PagedKV(k, v), x, x, torch.empty(0, dtype=torch.int64, device=DEV)) is None


# ------------------------------------------------------------------------------------------------ plan
def plan_reference(cached, new, table, free, n_free, page, T, n_pages):
    """The plan with Python loops; None when it is refused."""
    W = table.shape[1]
    table, free = table.copy(), free.copy()
    for c, n in zip(cached, new):
        if c < 0 or c > W * page:
            return -1
    back = [int(table[b, j]) for b in range(len(cached)) if new[b] < 0 for j in range(-(-cached[b] // page))]
    if n_free < 0 or n_free > n_pages or n_free + len(back) > n_pages:
        return -1
    if any(c + max(n, 0) > W * page for c, n in zip(cached, new)) or sum(max(n, 0) for n in new) > T:
        return -2
    free[n_free:n_free + len(back)] = back
    top = n_free + len(back)
    slots, row, ctx, first, out = [], [], [], [0], []
    for b, (c, n) in enumerate(zip(cached, new)):
        for j in range(-(-c // page), -(-(c + max(n, 0)) // page)):
            top -= 1
            if top < 0:
                return -2
            table[b, j] = free[top]
        for pos in range(c, c + max(n, 0)):
            slots.append(int(table[b, pos // page]) * page + pos % page)
            row.append(b)
            ctx.append(pos + 1)
        first.append(len(slots))
        out.append(0 if n < 0 else c + n)
    pad = T - len(slots)
    return table, free, top, out, slots + [-1] * pad, row + [-1] * pad, ctx + [0] * pad, first


def make_plan(paged, cached, new, page, T, slack=3, seed=0, width=None, in_place=True, n_pages=None):
    R = len(cached)
    have = [-(-c // page) for c in cached]
    width = width or max(-(-(c + max(n, 0)) // page) for c, n in zip(cached, new)) + 1
    need = sum(-(-(c + max(n, 0)) // page) - h for c, n, h in zip(cached, new, have))
    n_pages = n_pages or max(1, sum(have) + need + slack)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).numpy().astype(np.int32)
    table = np.full((R, width), -1, np.int32)
    at = 0
    for b in range(R):
        table[b, :have[b]] = order[at:at + have[b]]
        at += have[b]
    free = np.full(n_pages, -1, np.int32)
    free[: n_pages - at] = order[at:]
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    c = dev(cached)
    f = dev([n_pages - at])
    kw = {} if in_place else dict(cached_out=torch.empty_like(c), n_free_out=torch.empty_like(f))
    p = paged.PagePlan(cached=c, new_tokens=dev(new), table=dev(table), free=dev(free), n_free=f, page_size=page, max_tokens=T, **kw)
    return p, table, free, n_pages - at, n_pages


def check_plan(p, ref, cached=None):
    table, free, top, out, slots, row, ctx, first = ref
    assert int(p.status) == 0
    assert p.table.cpu().numpy().tolist() == table.tolist() and p.free.cpu().numpy().tolist() == free.tolist()
    assert int(p.n_free_out) == top and p.cached_out.tolist() == out and p.first.tolist() == first
    assert p.slots.tolist() == slots and p.row.tolist() == row and p.context.tolist() == ctx


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", ["one", "decode", "mixed", "prompts", "ends", "idle", "most", "full"])
def test_plan_against_loops(paged, case, in_place):
    rng = np.random.default_rng(3)
    page, pad = 16, 3
    if case == "one":
        cached, new = [0], [1]
    elif case == "decode":
        cached, new, page = list(range(60, 69)), [1] * 9, 64
    elif case == "mixed":
        cached, new = rng.integers(0, 700, 333).tolist(), rng.integers(-1, 40, 333).tolist()
    elif case == "prompts":
        cached, new = rng.integers(0, 20, 41).tolist(), rng.integers(0, 900, 41).tolist()
    elif case == "ends":
        cached, new, pad = [5, 0, 40, 16], [-1, -5, -1, -2147483648], 1
    elif case == "idle":
        cached, new, pad = [5, 0, 40, 16], [0] * 4, 2
    elif case == "most":
        cached, new = rng.integers(0, 50, 4096).tolist(), rng.integers(-1, 4, 4096).tolist()
    else:   # the pages that come back are the ones that are needed, to the last one
        cached, new = [160, 0, 33], [-1, 150, 15]
    T = max(1, sum(max(n, 0) for n in new) + pad)
    p, table, free, n_free, n_pages = make_plan(paged, cached, new, page, T, in_place=in_place, seed=7)
    if case == "full":
        p, table, free, n_free, n_pages = make_plan(paged, cached, new, page, T, in_place=in_place, seed=7, n_pages=13)
        assert n_free == 0
    ref = plan_reference(cached, new, table, free, n_free, page, T, n_pages)
    p.d3_page_plan()
    check_plan(p, ref)
    if not in_place:
        assert p.cached.tolist() == cached and int(p.n_free) == n_free
        p.d3_page_plan()             # nothing it reads has changed: the same again
        check_plan(p, ref)


def sum_plan(paged, in_place):
    """Three requests of 2^30 tokens each: their sums need more than 32 bits."""
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    c, f = dev([0, 0, 0]), dev([10])
    kw = {} if in_place else dict(cached_out=torch.empty_like(c), n_free_out=torch.empty_like(f))
    table = torch.full((3, 2 ** 20), -1, dtype=torch.int32, device=DEV)
    return paged.PagePlan(cached=c, new_tokens=dev([2 ** 30] * 3), table=table, free=dev(list(range(10))), n_free=f, page_size=1024,
                          max_tokens=50, **kw)


@pytest.mark.parametrize("why,code", [("pages", -2), ("width", -2), ("tokens", -2), ("cached", -1), ("length", -1), ("stack", -1),
                                      ("back", -1), ("sum", -2)])
@pytest.mark.parametrize("in_place", [True, False])
def test_plan_refuses_on_the_device_and_changes_nothing(paged, why, code, in_place):
    page, cached, new, kw = 16, [30, 100, 7], [3, 40, -1], {}
    if why == "width":
        kw["width"] = 8
    if why == "sum":
        p = sum_plan(paged, in_place)
    else:
        p = make_plan(paged, cached, new, page, 42 if why == "tokens" else 50, in_place=in_place, **kw)[0]
    if why == "pages":
        p.n_free.fill_(0)
        p.new_tokens[2] = 0
    if why == "cached":
        p.cached[1] = -1
    if why == "length":
        p.cached[1] = 16 * p.table.shape[1] + 1
    if why == "stack":
        p.n_free.fill_(p.free.numel() + 1)
    if why == "back":
        p.n_free.fill_(p.free.numel())
    kept = [t.clone() for t in (p.table, p.free, p.n_free, p.cached, p.new_tokens)]
    p.d3_page_plan()
    assert int(p.status) == code
    for t, k in zip((p.table, p.free, p.n_free, p.cached, p.new_tokens, p.n_free_out, p.cached_out), kept + [kept[2], kept[3]]):
        assert torch.equal(t, k)
    assert (p.slots == -1).all() and (p.row == -1).all() and (p.context == 0).all() and (p.first == 0).all()


def test_plan_reports_a_bad_page_of_a_request(paged):
    p, table, *_ = make_plan(paged, [20, 20], [1, 1], 16, 4)
    p.table[0, 1] = p.free.numel()
    p.d3_page_plan()
    assert int(p.status) == -1 and int(p.slots[0]) == -1
    assert int(p.slots[1]) == int(table[1, 1]) * 16 + 4 and p.context.tolist() == [21, 21, 0, 0]


# -------------------------------------------------------------------------------------------- together
class Serve:
    """A small serving loop over the three calls, with a dense 64-bit copy of every request."""

    def __init__(self, paged, kv, x, hq=8, hkv=2, dh=64, page=16, requests=6, n_pages=64, T=40, seed=0):
        self.P, self.hq, self.hkv, self.dh, self.page, self.T, self.R = paged, hq, hkv, dh, page, T, requests
        k, v = pool(n_pages, hkv, page, dh, kv, "token", seed)
        k.copy_(torch.full_like(k, math.nan)), v.copy_(torch.full_like(v, math.nan))
        self.cache = paged.PagedKV(k, v)
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
        self.new = dev([0] * requests)
        self.plan = paged.PagePlan(cached=dev([0] * requests), new_tokens=self.new,
                                   table=torch.full((requests, 12), -1, dtype=torch.int32, device=DEV), free=dev(list(range(n_pages))),
                                   n_free=dev([n_pages]), page_size=page, max_tokens=T)
        self.rope = paged.d3_rope_table(12 * page, dh)
        self.qkv = torch.zeros((T, hq + 2 * hkv, dh), dtype=x, device=DEV)
        self.q = torch.zeros((T, hq, dh), dtype=x, device=DEV)
        self.out = torch.zeros((T, hq, dh), dtype=x, device=DEV)
        self.lse = torch.zeros((T, hq), dtype=FP32, device=DEV)
        self.ws = paged.attention_workspace(self.cache, hq)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.kx, self.vx = [[] for _ in range(requests)], [[] for _ in range(requests)]
        self.g = torch.Generator(DEV).manual_seed(seed)

    def enqueue(self):
        hq, hkv, P = self.hq, self.hkv, self.P
        self.plan.d3_page_plan()
        P.d3_paged_append(self.cache, self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:], self.plan.slots, q=self.qkv[:, :hq], q_out=self.q,
                          rope=self.rope, context=self.plan.context, status=self.status)
        P.d3_paged_attention(self.cache, self.q, self.plan.table, self.plan.context, rows=self.plan.row, out=self.out, lse=self.lse,
                             workspace=self.ws, status=self.status)

    def inputs(self, new):
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.qkv.normal_(generator=self.g)
        self.out.fill_(11.0)

    def verify(self, new):
        torch.cuda.synchronize()
        assert int(self.plan.status) == 0 and int(self.status) == 0
        t = 0
        hq, hkv = self.hq, self.hkv
        for b, n in enumerate(new):
            if n < 0:
                self.kx[b], self.vx[b] = [], []
            for _ in range(max(n, 0)):
                ctx = torch.tensor([len(self.kx[b]) + 1], device=DEV)
                self.kx[b].append(rotated(self.qkv[t:t + 1, hq:hq + hkv], self.rope, ctx)[0].to(self.cache.dtype).double())
                self.vx[b].append(self.qkv[t, hq + hkv:].to(self.cache.dtype).double())
                q = rotated(self.qkv[t:t + 1, :hq], self.rope, ctx)[0].to(self.qkv.dtype)
                want, want_lse, tol, tol_lse = reference(q.double(), torch.stack(self.kx[b], 1), torch.stack(self.vx[b], 1),
                                                         self.dh ** -0.5, 2.0 ** -16)
                half = torch.finfo(self.out.dtype).eps / 2
                assert ((self.out[t].double() - want).abs() <= half * (want.abs() + tol) + tol + 1e-30).all(), (b, t)
                assert ((self.lse[t].double() - want_lse).abs() <= tol_lse).all()
                t += 1
        assert (self.out[t:] == 11.0).all()


STEPS = [[5, 0, 17, 0, 0, 1], [1, 3, 1, 0, 0, 1], [1, 1, -1, 20, 0, 1], [1, 1, 2, 1, 16, 1], [-1, 1, 1, 1, 1, -1], [31, 1, 1, 1, 1, 0],
         [1, 1, 1, 1, 1, 2], [0, 0, 0, 0, 0, 0], [1, 1, 1, 1, 1, 1]]


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (FP16, FP16), (BF16, FP32)], ids=["bf16", "fp16", "fp32"])
def test_a_serving_run_with_prompts_ends_and_reuse(paged, kv, x):
    s = Serve(paged, kv, x)
    for new in STEPS:
        s.inputs(new)
        s.enqueue()
        s.verify(new)


def test_a_captured_step_replays_with_other_lengths(paged):
    s = Serve(paged, BF16, BF16, seed=3)
    s.inputs(STEPS[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.enqueue()
    side.synchronize()
    s.verify(STEPS[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.enqueue()
    for new in STEPS[1:]:
        s.inputs(new)
        graph.replay()
        s.verify(new)


def test_calls_on_two_streams_with_workspaces_of_their_own(paged):
    sets = [make(paged, [3000, 50, 1200], 8, 2, 128, 16, BF16, BF16, seed=i) for i in range(2)]
    want = [paged.d3_paged_attention(c, q, t, n).clone() for c, t, q, n in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    spaces = [paged.attention_workspace(c, 8) for c, *_ in sets]
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for (c, t, q, n), st, ws, o in zip(sets, streams, spaces, outs):
            paged.d3_paged_attention(c, q, t, n, out=o, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_the_cache_of_a_loaded_model(paged):
    """d3_paged_view: attention over one block of a model's own pages, with the lengths of its slots."""
    from paper_2503_08524_b200 import binding as B
    from paper_2503_08524_b200 import inputs as I
    shape = I.TINY_GQA
    w = I.make_weights(shape, I.BASE_SEED + 5, device=DEV)
    m = B.D3Model(shape, w, 3, 128, 8, start_id=1, kv_fill=B.FILL_COPY, page_size=16, n_pages=120)
    m.poison_kv()
    lens = [37, 16]
    for slot, n in zip((2, 0), lens):
        m.d3_prefill(slot, I.prompt_tokens(shape, I.BASE_SEED, slot, n).numpy())
    m.d3_decode_step([2], [5], [1], 0.9)
    m.d3_sync()
    rows = [2, 0, -1]
    ctx = [m.d3_slot_pos(2), m.d3_slot_pos(0), 0]
    assert ctx[:2] == [38, 16]
    q = torch.empty((3, shape.n_q_heads, shape.head_dim), device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(2))
    for layer in (0, shape.n_layers - 1):
        cache, table = m.d3_paged_view(layer)
        assert table.shape == (3, 8) and cache.n_kv_heads == shape.n_kv_heads
        lse = torch.zeros((3, shape.n_q_heads), device=DEV)
        out = torch.zeros_like(q)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        paged.d3_paged_attention(cache, q, table, torch.tensor(ctx, dtype=torch.int32, device=DEV), out=out, lse=lse,
                                 rows=torch.tensor(rows, dtype=torch.int32, device=DEV), status=status)
        assert int(status) == 0
        check(out, lse, q, cache, table, ctx, rows=rows)
        for b, slot in ((0, 2), (1, 0)):      # the view shows what d3_read_kv reads
            for pos in (0, ctx[b] - 1):
                k, v = m.d3_read_kv(layer, slot, pos)
                page = int(table[slot, pos // 16])
                assert cache.k[page, :, pos % 16].float().flatten().tolist() == k.tolist()
                assert cache.v[page, :, pos % 16].float().flatten().tolist() == v.tolist()
    for bad in (-1, shape.n_layers):
        with pytest.raises(B.D3Error):
            m.d3_paged_view(bad)
    m.close()
