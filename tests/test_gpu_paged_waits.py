"""Waits of the paged attention that run out: nothing faults, the call says so, the next one is right."""
import pytest
import torch

from paper_2503_08524_b200.binding import ETIMEOUT
from test_gpu_paged import BF16, DEV, E4M3, FP32, check, make, paged  # noqa: F401  (paged: a fixture)

pytestmark = pytest.mark.gpu
LIMIT_NS = 3_000_000


@pytest.fixture
def limit(paged):
    yield paged.d3_paged_set_wait_ns
    paged.d3_paged_stall_next(0)
    paged.d3_paged_set_wait_ns(2_000_000_000)


# how the rows are dealt out: (contexts, query heads, kv heads, entries of a table row; 0: as many as the longest row needs).  The
# first CTA has several stages in each.
DEALT = {"cluster": ([2000, 1000, 1999, 64], 8, 4, 0), "whole": ([600] * 12, 16, 8, 0), "cut, few rows": ([9000, 3, 900, 0, 2500], 8, 2, 4000),
         "cut, many rows": ([9000] + [(31 * i) % 90 for i in range(139)], 4, 2, 4000)}


@pytest.mark.parametrize("kv,x", [(BF16, BF16), (BF16, FP32), (E4M3, BF16)], ids=["bf16", "bf16-fp32", "e4m3-bf16"])
@pytest.mark.parametrize("what", ["STALL_COPIES", "STALL_SUMS"])
@pytest.mark.parametrize("dealt", list(DEALT))
def test_attention_waits_that_run_out_are_reported(paged, limit, dealt, what, kv, x):
    contexts, hq, hkv, width = DEALT[dealt]
    cache, table, q, ctx = make(paged, contexts, hq, hkv, 128, 16, kv, x, seed=19)
    if width:
        wide = torch.full((len(contexts), width), -1, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        table = wide
    ws, status = paged.attention_workspace(cache, hq), torch.zeros(1, dtype=torch.int32, device=DEV)
    call = lambda: paged.d3_paged_attention(cache, q, table, ctx, with_lse=True, workspace=ws, status=status)  # noqa: E731
    out, lse = call()
    assert int(status) == 0
    check(out, lse, q, cache, table, contexts)
    limit(LIMIT_NS)
    paged.d3_paged_stall_next(getattr(paged, what))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    call()
    end.record()
    torch.cuda.synchronize()
    assert int(status) == ETIMEOUT
    assert 2.5 < begin.elapsed_time(end) < 500.0       # it waited its limit (and a second one, for a cluster's first CTA), not forever
    status.zero_()
    again = call()                                     # the drill was for one call; the limit is far above what a wait takes
    assert int(status) == 0 and torch.equal(again[0], out) and torch.equal(again[1], lse)
    paged.d3_paged_stall_next(paged.STALL_SUMS)
    paged.d3_paged_stall_next(0)                       # taken back
    again = call()
    assert int(status) == 0 and torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dealt", ["cluster", "whole", "cut, few rows"])
def test_attention_waits_do_not_count_the_call_before(paged, limit, dealt):
    """The limit is that of the call's own waits: a call may start its CTAs while the one before it, some milliseconds long, runs."""
    contexts, hq, hkv, width = DEALT[dealt]
    cache, table, q, ctx = make(paged, contexts, hq, hkv, 128, 16, BF16, BF16, seed=19)
    if width:
        wide = torch.full((len(contexts), width), -1, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        table = wide
    ws, status = paged.attention_workspace(cache, hq), torch.zeros(1, dtype=torch.int32, device=DEV)
    call = lambda: paged.d3_paged_attention(cache, q, table, ctx, with_lse=True, workspace=ws, status=status)  # noqa: E731
    out, lse = call()
    # long and on one multiprocessor: a plan in which all of 100 long requests end
    pages = 16384
    i32 = dict(dtype=torch.int32, device=DEV)
    plan = paged.PagePlan(cached=torch.full((100,), 16 * pages, **i32), new_tokens=torch.full((100,), -1, **i32),
                          table=torch.arange(100 * pages, **i32).view(100, pages), free=torch.zeros(100 * pages, **i32),
                          n_free=torch.zeros(1, **i32), page_size=16, max_tokens=8, cached_out=torch.zeros(100, **i32),
                          n_free_out=torch.zeros(1, **i32))
    plan.d3_page_plan()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    plan.d3_page_plan()
    end.record()
    torch.cuda.synchronize()
    limit(500_000)
    assert int(plan.status) == 0 and begin.elapsed_time(end) > 2.0      # much longer than the limit
    plan.d3_page_plan()
    again = call()
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(again[0], out) and torch.equal(again[1], lse)
