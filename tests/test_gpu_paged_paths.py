"""The paged operators where one call's leftovers could reach the next: workspaces, captured calls, pages given back."""
import pytest
import torch

from test_gpu_paged import BF16, DEV, make, make_plan, paged  # noqa: F401  (paged: a fixture)

pytestmark = pytest.mark.gpu


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
