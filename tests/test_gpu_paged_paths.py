"""The paged operators where one call's leftovers could reach the next: workspaces, captured calls, pages given back."""
import pytest
import torch

from test_gpu_paged import (BF16, DEV, E4M3, FP16, FP32, check, check_plan, make, make_plan, paged, plan_reference,  # noqa: F401
                            pool)

pytestmark = pytest.mark.gpu


def widened(table, width=4000):
    """A table with room for more than any row has: rows are then cut between CTAs and joined through the workspace."""
    wide = torch.full((table.shape[0], width), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    return wide


def parts_written(ws, dh, fill):
    """Whether pieces of rows were left in a workspace that held `fill` (they lie in front of its last 192 * 16 bytes)."""
    return bool((ws[: 2 * 192 * 16 * dh * 4] != fill).any())


# (contexts, rows): few rows, more rows than a warp sums up; all with rows that are cut
CUTS = {"few": [9000, 3, 900, 0, 2500], "many": [9000] + [(31 * i) % 90 for i in range(139)]}


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (E4M3, FP16)], ids=["bf16", "bf16-fp32", "e4m3-fp16"])
@pytest.mark.parametrize("rows", list(CUTS))
def test_attention_cut_rows_ignore_what_the_workspace_holds(paged, kv, x, rows):
    contexts = CUTS[rows]
    cache, table, q, ctx = make(paged, contexts, 16, 4, 128, 32, kv, x, seed=11)
    table = widened(table)
    ws = paged.attention_workspace(cache, 16)
    first = None
    for fill in (0, 255, 85):
        ws.fill_(fill)
        out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True, workspace=ws)
        assert parts_written(ws, 128, fill)
        if first is None:
            first = (out.clone(), lse.clone())
            check(out, lse, q, cache, table, contexts)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("rows", list(CUTS))
def test_attention_cut_rows_on_two_streams(paged, rows):
    sets = [make(paged, CUTS[rows][::d], 8, 2, 128, 16, BF16, BF16, seed=i) for i, d in enumerate((1, -1))]
    sets = [(c, widened(t), q, n) for c, t, q, n in sets]
    want = [paged.d3_paged_attention(c, q, t, n).clone() for c, t, q, n in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    spaces = [paged.attention_workspace(c, 8) for c, *_ in sets]
    outs = [torch.zeros_like(w) for w in want]
    for ws in spaces:
        ws.fill_(255)
    torch.cuda.synchronize()
    for _ in range(20):
        for (c, t, q, n), st, ws, o in zip(sets, streams, spaces, outs):
            paged.d3_paged_attention(c, q, t, n, out=o, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for o, w, ws in zip(outs, want, spaces):
        assert torch.equal(o, w) and parts_written(ws, 128, 255)


@pytest.mark.parametrize("rows", [6, 140])
def test_attention_cut_rows_captured_and_replayed_with_other_lengths(paged, rows):
    """One workspace through replays in which the long row, the one that is cut, stands first, last, nowhere."""
    top = 9000
    k, v = pool(2 * (top // 32 + 1) + rows, 2, 32, 128, BF16, seed=5)
    cache = paged.PagedKV(k, v)
    g = torch.Generator().manual_seed(rows)
    table = torch.randint(0, cache.n_pages, (rows, 2000), generator=g, dtype=torch.int32).to(DEV)     # (rows may share pages)
    q = torch.empty((rows, 8, 128), dtype=BF16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(6))
    ctx = torch.full((rows,), 5, dtype=torch.int32, device=DEV)
    ws = paged.attention_workspace(cache, 8)
    out, lse = torch.zeros_like(q), torch.zeros((rows, 8), device=DEV)
    call = lambda: paged.d3_paged_attention(cache, q, table, ctx, out=out, lse=lse, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    short = [(13 * i) % 70 for i in range(rows)]
    cases = [[top] + short[1:], short[:-1] + [top], short, [0] * rows, [top, top - 1] + [0] * (rows - 2), [1] * rows]
    for lengths in cases + cases[::-1]:
        ctx.copy_(torch.tensor(lengths, dtype=torch.int32))
        ws.fill_(255)
        graph.replay()
        if max(lengths) == top:
            assert parts_written(ws, 128, 255)
        check(out, lse, q, cache, table, lengths)
        bits, l_bits = out.clone(), lse.clone()
        call()
        assert torch.equal(out, bits) and torch.equal(lse, l_bits)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("what", ["tokens", "width", "both"])
def test_plan_with_sums_of_64_bits(paged, what, in_place):
    """Sizes beyond which the sums over the requests are kept in 64 bits."""
    page, cached, new = 16, [30, 0, 100, 7, 250], [3, 500, 40, -1, 0]
    T = 2 ** 18 + 3 if what != "width" else 600
    p, table, free, n_free, n_pages = make_plan(paged, cached, new, page, T, in_place=in_place, seed=3,
                                                width=2 ** 18 + 1 if what != "tokens" else None)
    ref = plan_reference(cached, new, table, free, n_free, page, T, n_pages)
    p.d3_page_plan()
    check_plan(p, ref)


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, -2 ** 31, "n_pages"])
@pytest.mark.parametrize("requests", [3, 300])
def test_plan_reports_a_bad_page_that_comes_back(paged, bad, requests):
    """An ended request whose row holds no page id inside its length: the call that takes it back says so, and so does the one that
    hands it out; no slot is made of it."""
    cached, new = [40, 20, 33] + [5] * (requests - 3), [-1, 0, 0] + [0] * (requests - 3)
    p, table, free, n_free, n_pages = make_plan(paged, cached, new, 16, 600, slack=0)
    bad = n_pages if bad == "n_pages" else bad
    p.table[0, 1] = bad
    p.d3_page_plan()
    assert int(p.status) == -1
    assert int(p.n_free) == 3 and p.free[:3].tolist() == [int(table[0, 0]), bad, int(table[0, 2])]
    assert p.cached.tolist() == [0] + cached[1:]
    p.status.zero_()
    p.new_tokens.zero_()
    p.new_tokens[1] = 13                       # 20 -> 33: one page, the last that came back
    p.d3_page_plan()
    assert int(p.status) == 0 and int(p.table[1, 2]) == int(table[0, 2])
    p.new_tokens[1] = 16                       # 33 -> 49: the bad one
    p.d3_page_plan()
    assert int(p.status) == -1
    assert p.slots[:16].tolist() == [int(table[0, 2]) * 16 + i for i in range(1, 16)] + [-1]


def small(paged, kv=BF16):
    cache, table, q, ctx = make(paged, [40, 7], 8, 2, 64, 16, kv, BF16, seed=2)
    new = torch.ones((2, 2, 64), dtype=BF16, device=DEV)
    slots = torch.tensor([3, 40], device=DEV)
    rope = paged.d3_rope_table(64, 64)
    return cache, table, q, ctx, new, slots, rope


def test_written_tensors_are_known_to_autograd(paged):
    """What a call writes into counts as changed: a graph that had saved it says so in its backward pass."""
    cache, table, q, ctx, new, slots, rope = small(paged)
    p = make_plan(paged, [20, 20], [1, 1], 16, 4)[0]
    q_out, out, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((2, 8), device=DEV)
    written = {"append": (cache.k, cache.v, q_out), "attention": (out, lse),
               "plan": (p.table, p.free, p.cached_out, p.n_free_out, p.slots, p.row, p.context, p.first)}
    calls = {"append": lambda: paged.d3_paged_append(cache, new, new, slots, q=q, q_out=q_out, rope=rope, context=ctx),
             "attention": lambda: paged.d3_paged_attention(cache, q, table, ctx, out=out, lse=lse), "plan": p.d3_page_plan}
    for name, call in calls.items():
        w = [torch.ones((), device=DEV, requires_grad=True) for _ in written[name]]
        y = [t * s for t, s in zip(written[name], w)]
        before = [t._version for t in written[name]]
        call()
        assert all(t._version > v for t, v in zip(written[name], before)), name
        for z in y:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                z.float().sum().backward()
    with torch.inference_mode():               # (tensors without a count)
        cache, table, q, ctx, new, slots, rope = small(paged)
        paged.d3_paged_append(cache, new, new, slots, q=q, q_out=q, rope=rope, context=ctx)
        got = paged.d3_paged_attention(cache, q, table, ctx, out=torch.empty_like(q), with_lse=True)
        make_plan(paged, [20, 20], [1, 1], 16, 4)[0].d3_page_plan()
    assert got[0].isfinite().all()
