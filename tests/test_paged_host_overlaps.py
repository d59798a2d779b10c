"""Buffers of one call of the paged operators that overlap: refused on the host, before anything is enqueued (no GPU)."""
import ctypes as C
import itertools
import random

import pytest
import torch

from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import paged as P
from test_paged_host import append_args, kv_args

BASE, GAP = 1 << 24, 1 << 20          # addresses that no call dereferences on the host
NAMES = ("cached_dev", "new_tokens_dev", "table_dev", "free_dev", "n_free_dev", "cached_out_dev", "n_free_out_dev", "first_dev",
         "slots_dev", "row_dev", "context_dev", "status_dev")
READ = ("cached_dev", "new_tokens_dev", "n_free_dev")
R, PAGES, WIDTH, T, STRIDE = 5, 40, 6, 12, 10
SIZE = dict(cached_dev=4 * R, new_tokens_dev=4 * R, table_dev=4 * (STRIDE * (R - 1) + WIDTH), free_dev=4 * PAGES, n_free_dev=4,
            cached_out_dev=4 * R, n_free_out_dev=4, first_dev=4 * R + 4, slots_dev=8 * T, row_dev=4 * T, context_dev=4 * T, status_dev=4)
GOOD = B.ECUDA                        # accepted: the launch itself fails where there is no device
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would run")


def plan(**kw):
    at = {n: BASE + i * GAP for i, n in enumerate(NAMES)}
    at.update(kw)
    a = P.PagePlanArgs(C.sizeof(P.PagePlanArgs), R, 16, PAGES, WIDTH, T, STRIDE, *[at[n] for n in NAMES])
    return B.LIB.d3_page_plan(C.byref(a), None)


def where(n):
    return BASE + NAMES.index(n) * GAP


@no_device
def test_plans_whose_buffers_lie_apart_are_accepted():
    assert plan() == GOOD and plan(status_dev=None) == GOOD
    assert plan(cached_out_dev=where("cached_dev"), n_free_out_dev=where("n_free_dev")) == GOOD
    t = where("table_dev")
    for n in NAMES:                   # before, behind, and between the rows of the table
        if n == "table_dev":
            continue
        before, behind = (t - SIZE[n]) // 16 * 16, t + (SIZE["table_dev"] + 15) // 16 * 16
        assert plan(**{n: before}) == GOOD and plan(**{n: behind}) == GOOD, n
        if SIZE[n] <= 4 * (STRIDE - WIDTH) and n not in ("slots_dev", "row_dev", "context_dev"):
            assert plan(**{n: t + 4 * (STRIDE * 2 + WIDTH)}) == GOOD, n
    assert plan(cached_dev=where("new_tokens_dev")) == GOOD              # both are read


@pytest.mark.parametrize("one,other", list(itertools.combinations(NAMES, 2)))
def test_plans_whose_buffers_overlap_are_refused(one, other):
    if one in READ and other in READ:
        return
    in_place = {one, other} in ({"cached_dev", "cached_out_dev"}, {"n_free_dev", "n_free_out_dev"})
    wide = [n for n in (one, other) if n in ("slots_dev", "row_dev", "context_dev")]
    for moved, still in ((one, other), (other, one)):
        step = 16 if moved in wide else 4
        first = -(SIZE[moved] - 4) // step * step
        for off in {0, first, (SIZE[still] - 1) // step * step, step}:
            if off == 0 and in_place or not -SIZE[moved] < off < SIZE[still]:
                continue
            if "table_dev" in (one, other):   # not where only the gap between two rows is met
                lo, n = (off, SIZE[moved]) if still == "table_dev" else (-off, SIZE[still])
                if not any(r * STRIDE * 4 < lo + n and lo < r * STRIDE * 4 + WIDTH * 4 for r in range(R)):
                    continue
            assert plan(**{moved: where(still) + off}) == B.EINVAL, (moved, still, off)


@pytest.mark.parametrize("bad", [
    dict(struct_size=0), dict(n_requests=0), dict(n_requests=4097), dict(page_size=17), dict(page_size=0), dict(n_pages=0),
    dict(table_width=0), dict(max_tokens=0), dict(table_stride=WIDTH - 1), dict(table_width=1 << 27, table_stride=1 << 27),
    *[{n: None} for n in NAMES if n != "status_dev"], *[{n: where(n) + 8} for n in ("slots_dev", "row_dev", "context_dev")],
    dict(table_dev=where("table_dev") + 1), dict(status_dev=where("status_dev") + 2)], ids=str)
def test_plans_over_buffers_apart_are_refused_for_one_reason(bad):
    a = P.PagePlanArgs(C.sizeof(P.PagePlanArgs), R, 16, PAGES, WIDTH, T, STRIDE, *[where(n) for n in NAMES])
    for k, v in bad.items():
        setattr(a, k, v)
    assert B.LIB.d3_page_plan(C.byref(a), None) == B.EINVAL


def cells(n, s, dh, base=0):
    return {base + sum(i * t for i, t in zip(ix, s)) + d for ix in itertools.product(*[range(c) for c in n]) for d in range(dh)}


def append(kv, **kw):
    """An accepted call would go on to a launch: only where that cannot be."""
    return B.LIB.d3_paged_append(C.byref(kv), C.byref(append_args(k_dev=8 * BASE, v_dev=9 * BASE, slots_dev=10 * BASE, context_dev=11 * BASE,
                                                                  rope_dev=12 * BASE, **kw)), None)


@no_device
def test_pools_whose_k_and_v_overlap_are_refused():
    """Against sets of addresses: V anywhere around K, by layouts that lie close, interleave and leave gaps."""
    rng = random.Random(5)
    dh, n = 32, (3, 2, 16)           # pages, kv heads, positions
    for s in ((1024, 512, 32), (1024, 32, 64), (2048, 1024, 64), (32, 96, 192), (4096, 64, 256), (8192, 2048, 64)):
        far = sum((c - 1) * t for c, t in zip(n, s)) + dh
        offsets = [0, s[0], s[1], s[2], -s[0], 32, -32, 64, s[0] * 3, s[1] * 2, s[2] * 16, far, -far] + \
            [8 * rng.randint(-far // 8 - 4, far // 8 + 4) for _ in range(60)]
        k_cells = cells(n, s, dh)
        seen = set()
        for off in offsets:
            kv = kv_args(n_pages=3, n_kv_heads=2, head_dim=dh, page_stride=s[0], head_stride=s[1], token_stride=s[2], k_dev=2 * BASE,
                         v_dev=2 * BASE + 2 * off)
            meet = not k_cells.isdisjoint(cells(n, s, dh, off))
            seen.add(meet)
            assert append(kv, q_dev=None, k_token_stride=64, k_head_stride=32, v_token_stride=64, v_head_stride=32) == \
                (B.EINVAL if meet else GOOD), (s, off)
        assert seen == {True, False}


@no_device
def test_q_out_beside_q_or_q_itself_but_nowhere_between():
    kv = kv_args(k_dev=2 * BASE, v_dev=3 * BASE)                      # head dim 64, 5 tokens of 4 heads
    for st, sh in ((256, 64), (512, 64), (512, 128), (64, 320)):
        q_cells = cells((5, 4), (st, sh), 64)
        for off in (0, 64, -64, 8, 128, 256, -256, 1280, 320, 5 * st, -5 * st, 4 * sh, 24):
            meet = off != 0 and not q_cells.isdisjoint(cells((5, 4), (st, sh), 64, off))
            kw = dict(q_dev=4 * BASE, q_out_dev=4 * BASE + 2 * off, q_token_stride=st, q_head_stride=sh, q_out_token_stride=st,
                      q_out_head_stride=sh)
            assert append(kv, **kw) == (B.EINVAL if meet else GOOD), (st, sh, off)
