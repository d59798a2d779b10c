"""Calls of the paged operators that their documentation allows, at its edges: layouts, strides, sizes, shared workspaces.

Tolerances are those of test_gpu_paged.py.
"""
import math

import pytest
import torch

from test_gpu_paged import BF16, DEV, E4M3, FP16, FP32, check, check_plan, make, paged, plan_reference, rotated, tables  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (E4M3, BF16)], ids=["bf16", "bf16-fp32", "e4m3-bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 4.0])
def test_attention_scales(paged, scale, kv, x):
    contexts = [300, 17, 0, 64]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 64, 16, kv, x, seed=3, q_std=0.5)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, scale=scale, with_lse=True)
    check(out, lse, q, cache, table, contexts, scale=scale)


@pytest.mark.parametrize("order", ["page, kv", "page, token, kv", "page, token, head, kv"])
def test_keys_and_values_interleaved_in_one_tensor(paged, order):
    """The layouts that keep a page's (a token's, a head's) K and V side by side: appended to and read."""
    n_pages, hkv, page, dh = 12, 2, 16, 64
    shape, k_of = {"page, kv": ((n_pages, 2, hkv, page, dh), lambda t, i: t[:, i]),
                   "page, token, kv": ((n_pages, page, 2, hkv, dh), lambda t, i: t[:, :, i].permute(0, 2, 1, 3)),
                   "page, token, head, kv": ((n_pages, page, hkv, 2, dh), lambda t, i: t[:, :, :, i].permute(0, 2, 1, 3))}[order]
    g = torch.Generator(DEV).manual_seed(1)
    both = torch.full(shape, math.nan, dtype=BF16, device=DEV)
    cache = paged.PagedKV(k_of(both, 0), k_of(both, 1))
    n = 5 * page - 3
    k, v = (torch.empty((n, hkv, dh), dtype=BF16, device=DEV).normal_(generator=g) for _ in range(2))
    ids = [7, 0, 11, 3, 9]
    table = torch.tensor([ids], dtype=torch.int32, device=DEV)
    slots = torch.tensor([ids[i // page] * page + i % page for i in range(n)], device=DEV)
    paged.d3_paged_append(cache, k, v, slots)
    for t, new in ((cache.k, k), (cache.v, v)):
        assert torch.equal(t[torch.tensor(ids)].permute(0, 2, 1, 3).reshape(-1, hkv, dh)[:n], new)
    assert int(both.isnan().sum()) == both.numel() - 2 * n * hkv * dh
    q = torch.empty((1, 8, dh), dtype=BF16, device=DEV).normal_(generator=g)
    out, lse = paged.d3_paged_attention(cache, q, table, torch.tensor([n], dtype=torch.int32, device=DEV), with_lse=True)
    check(out, lse, q, cache, table, [n])


def test_inputs_that_are_broadcast(paged):
    contexts = [100, 33, 64]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 64, 16, BF16, BF16, seed=4)
    for one in (q[:1].expand(3, 8, 64), q[:, :1].expand(3, 8, 64), q[:1, :1].expand(3, 8, 64)):
        assert 0 in one.stride()
        out, lse = paged.d3_paged_attention(cache, one, table, ctx, with_lse=True)
        check(out, lse, one, cache, table, contexts)
    slots, rope = torch.tensor([5, 21, 40], device=DEV), paged.d3_rope_table(128, 64)
    k, q_out = q[:1, :1].expand(3, 2, 64), torch.zeros_like(q)
    paged.d3_paged_append(cache, k, k, slots, q=q[:1].expand(3, 8, 64), q_out=q_out, rope=rope, context=ctx)
    for t, want in ((cache.k, rotated(k, rope, ctx).to(BF16)), (cache.v, k)):
        assert torch.equal(t.permute(0, 2, 1, 3)[slots // 16, slots % 16], want)
    assert torch.equal(q_out, rotated(q[:1].expand(3, 8, 64), rope, ctx).to(BF16))


def test_tables_that_are_views(paged):
    """Rows of a wider table, every second row of one, and a plan over such a table: what lies between the rows stays."""
    contexts = [300, 17, 64]
    cache, table, q, ctx = make(paged, contexts, 8, 2, 64, 16, BF16, BF16, seed=4)
    big = torch.full((6, 40), -9, dtype=torch.int32, device=DEV)
    view = big[::2, 3:3 + table.shape[1]]
    view.copy_(table)
    out, lse = paged.d3_paged_attention(cache, q, view, ctx, with_lse=True)
    check(out, lse, q, cache, table, contexts)
    cached, new = [30, 7, 100], [40, -1, 13]
    start = tables(cached, 16, 30, 2, spare=3)
    used = set(start.flatten().tolist()) - {-1}
    free = [p for p in range(30) if p not in used]
    big.fill_(-9)
    view = big[::2, 5:5 + start.shape[1]]
    view.copy_(start)
    stack = torch.tensor(free + [-1] * (30 - len(free)), dtype=torch.int32, device=DEV)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    ref = plan_reference(cached, new, start.cpu().numpy(), stack.cpu().numpy(), len(free), 16, 60, 30)
    p = paged.PagePlan(cached=dev(cached), new_tokens=dev(new), table=view, free=stack, n_free=dev([len(free)]), page_size=16, max_tokens=60)
    p.d3_page_plan()
    check_plan(p, ref)
    assert int((big != -9).sum()) == start.numel()


def test_attention_of_no_rows(paged):
    cache, table, q, ctx = make(paged, [40], 8, 2, 64, 16, BF16, BF16, seed=4)
    out, lse = paged.d3_paged_attention(cache, q[:0], table, ctx[:0], rows=ctx[:0], with_lse=True)
    assert out.shape == (0, 8, 64) and lse.shape == (0, 8)


@pytest.mark.parametrize("rows_map", [False, True])
def test_attention_of_the_most_rows(paged, rows_map):
    """65535 rows of 0 to 3 positions."""
    n, dh, hq, hkv, page = 65535, 32, 2, 1, 16
    g = torch.Generator(DEV).manual_seed(6)
    k, v = (torch.empty((n, hkv, page, dh), dtype=BF16, device=DEV).normal_(generator=g) for _ in range(2))
    cache = paged.PagedKV(k, v)
    q = torch.empty((n, hq, dh), dtype=BF16, device=DEV).normal_(generator=g)
    ctx = torch.randint(0, 4, (n,), generator=g, device=DEV, dtype=torch.int32)
    table = torch.randperm(n, generator=g, device=DEV).int()[:, None].contiguous()
    rows = torch.randint(-1, n, (n,), generator=g, device=DEV, dtype=torch.int32) if rows_map else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((n, hq), 7.0, device=DEV)
    paged.d3_paged_attention(cache, q, table, ctx, rows=rows, out=out, lse=lse, status=status)
    assert int(status) == 0
    at = torch.arange(n, device=DEV) if rows is None else rows.long()
    live, some = at >= 0, ctx > 0
    ids = table[at.clamp(min=0), 0].long()
    kd, vd = k[ids, 0, :4].double(), v[ids, 0, :4].double()
    s = torch.einsum("bhd,btd->bht", q.double(), kd) * dh ** -0.5
    s = s.masked_fill(torch.arange(4, device=DEV) >= ctx[:, None, None], -math.inf)
    p = torch.softmax(s[some], -1)
    # (as in `reference`: errors of the scores, two bf16 terms, sums and joining, the exponentials)
    d = (dh + 8) * 2.0 ** -23 * dh ** -0.5 * torch.einsum("bhd,btd->bht", q[some].double().abs(), kd[some].abs()).amax(-1, keepdim=True)
    E = 2 * d + 2.0 ** -16 + 200 * 2.0 ** -23 + 2.0 ** -20
    want, tol = p @ vd[some], E * (p @ vd[some].abs())
    keep = live[some]
    assert ((out[some].double() - want).abs() <= 2.0 ** -8 * (want.abs() + tol) + tol)[keep].all()
    want_lse = torch.logsumexp(s[some], -1)
    assert ((lse[some].double() - want_lse).abs() <= E.squeeze(-1) + want_lse.abs() * 2.0 ** -22)[keep].all()
    assert (out[live & ~some] == 0).all() and (lse[live & ~some] == -math.inf).all()
    assert (out[~live] == 7.0).all() and (lse[~live] == 7.0).all()


def test_attention_positions_up_to_the_largest(paged):
    """A context of almost 2^31 positions, over pages that repeat: the result is that of one round of them, lse + log(rounds)."""
    page, dh, period = 1024, 32, 7
    g = torch.Generator(DEV).manual_seed(8)
    k, v = (torch.empty((period, 1, page, dh), dtype=FP16, device=DEV).normal_(generator=g) for _ in range(2))
    k.mul_(0.05)
    cache = paged.PagedKV(k, v)
    width = (2 ** 31 - 1 - 1024) // page // period * period
    table = (torch.arange(width, device=DEV) % period).int()[None].contiguous()
    q = torch.empty((1, 2, dh), dtype=FP16, device=DEV).normal_(generator=g)
    ctx = torch.tensor([width * page], dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True, status=status)
    assert int(status) == 0
    s = torch.einsum("hd,td->ht", q[0].double(), k.double().reshape(-1, dh)) * dh ** -0.5
    want = torch.softmax(s, -1) @ v.double().reshape(-1, dh)
    # a lane adds up one weight of 16 positions after another (the products' sums grow alike): all of them half a step off
    steps = width * page / 16 / (148 * 10)
    E = steps * 2.0 ** -24
    assert ((lse[0].double() - torch.logsumexp(s, -1) - math.log(width // period)).abs() <= E + 30 * 2.0 ** -23).all()
    assert ((out[0].double() - want).abs() <= 2 * E * v.double().abs().mean() * 1.1 + 2.0 ** -11).all()


def test_two_captured_steps_share_a_workspace(paged):
    """Graphs of two calls over one workspace, replayed in turn on one stream; both calls cut rows."""
    sets = [make(paged, c, 8, 2, 128, 16, BF16, BF16, seed=i) for i, c in enumerate(([5000, 50, 1200], [64, 7000]))]
    wide = []
    for c, t, q, n in sets:
        w = torch.full((t.shape[0], 3000), -1, dtype=torch.int32, device=DEV)
        w[:, :t.shape[1]] = t
        wide.append(w)
    ws = paged.attention_workspace(sets[0][0], 8)
    want = [paged.d3_paged_attention(c, q, w, n) for (c, _, q, n), w in zip(sets, wide)]
    outs = [torch.zeros_like(x) for x in want]
    graphs = []
    for (c, _, q, n), w, o in zip(sets, wide, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            paged.d3_paged_attention(c, q, w, n, out=o, workspace=ws)
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1, 0, 0):
        outs[i].zero_()
        ws.fill_(255)
        for j in (1 - i, i):
            graphs[j].replay()
        assert torch.equal(outs[i], want[i]) and torch.equal(outs[1 - i], want[1 - i])
