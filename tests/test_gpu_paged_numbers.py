"""Attention over a paged cache where its numbers could lose bits or leave the finite range.

Tolerances are those of test_gpu_paged.py (`reference` there), with the term of the weights of two
fp16 numbers, 2^-21, under every 8-bit cache.
"""
import math

import pytest
import torch

from test_gpu_paged import BF16, DEV, E4M3, FP16, FP32, check, make, paged, reference  # noqa: F401  (paged: a fixture)

pytestmark = pytest.mark.gpu


def close(out, lse, q, k, v, scale, terms=2.0 ** -21):
    """out, lse [rows][hq](..) against the 64-bit form over k, v [kv head][n][dim]."""
    half = torch.finfo(out.dtype).eps / 2
    for b in range(q.shape[0]):
        want, want_lse, tol, tol_lse = reference(q[b].double(), k, v, scale, terms)
        err = (out[b].double() - want).abs()
        allowed = half * (want.abs() + tol) + tol
        assert (err <= allowed).all(), (b, float((err / allowed).max()))
        assert ((lse[b].double() - want_lse).abs() <= tol_lse).all(), b


@pytest.mark.parametrize("x", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("hq", [1, 16])
def test_attention_8_bit_weights_that_nearly_cancel(paged, x, dh, hq):
    """Two positions of nearly equal weights and opposite values: what a weight was rounded to shows in the result."""
    rows = 64
    k, v = (torch.zeros((rows, 1, 16, dh), device=DEV).to(E4M3) for _ in range(2))
    k[:, 0, 0, 0], k[:, 0, 1, 0] = 1.0, 1.125
    v[:, 0, 0], v[:, 0, 1] = 1.0, -1.0
    cache = paged.PagedKV(k, v)
    q = torch.zeros((rows, hq, dh), dtype=x, device=DEV)
    q[:, :, 0] = torch.linspace(0.01, 0.2, rows * hq, device=DEV).view(rows, hq).to(x)
    table = torch.arange(rows, dtype=torch.int32, device=DEV)[:, None].contiguous()
    ctx = torch.full((rows,), 2, dtype=torch.int32, device=DEV)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, scale=1.0, with_lse=True)
    close(out, lse, q, k[0, :, :2].double(), v[0, :, :2].double(), 1.0)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("hq", [4, 32])
@pytest.mark.parametrize("reach", [20, 30, 36])
def test_attention_8_bit_small_parts_of_a_query_count(paged, dh, hq, reach):
    """A query whose largest entry meets only zeros, the others 2^-reach of it and up (fp16 holds those numbers when the largest
    is brought to 2^14): they alone make the scores."""
    n, g = 200, torch.Generator(DEV).manual_seed(reach + dh)
    cache, table, q, ctx = make(paged, [n], hq, 2, dh, 16, E4M3, BF16, seed=dh, scales="none")
    cache.k[..., 3] = 0.0
    low = 2.0 ** (20 - reach)
    q.copy_((torch.randint(-127, 128, q.shape, generator=g, device=DEV) * low).to(BF16))
    q[:, :, 3] = 2.0 ** 20
    scale = 1.0 / (low * 127 * 30 * dh ** 0.5)
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, scale=scale, with_lse=True)
    ids = table[0].tolist()[: -(-n // 16)]
    k, v = (torch.stack([t[p].float() for p in ids]).double().permute(1, 0, 2, 3).reshape(2, -1, dh)[:, :n] for t in (cache.k, cache.v))
    close(out, lse, q, k, v, scale)


def test_attention_8_bit_queries_below_the_normal_numbers(paged):
    n, dh, g = 100, 64, torch.Generator(DEV).manual_seed(5)
    cache, table, q, ctx = make(paged, [n], 8, 2, dh, 16, E4M3, BF16, seed=8, scales="none")
    q.copy_((torch.randint(-127, 128, q.shape, generator=g, device=DEV) * 2.0 ** -60 * 2.0 ** -73).to(BF16))
    assert 0 < float(q.float().abs().max()) < 2.0 ** -126
    out, lse = paged.d3_paged_attention(cache, q, table, ctx, scale=1e36, with_lse=True)
    ids = table[0].tolist()[: -(-n // 16)]
    k, v = (torch.stack([t[p].float() for p in ids]).double().permute(1, 0, 2, 3).reshape(2, -1, dh)[:, :n] for t in (cache.k, cache.v))
    close(out, lse, q, k, v, 1e36)


# whole rows, a cluster for each row, rows cut between CTAs (by the room in the table)
MODES = {"whole": ([70, 30], 0), "cluster": ([700, 300], 0), "cut": ([3000, 300], 4000)}


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("kv,x", [(BF16, BF16), (FP16, FP16), (BF16, FP32)], ids=["bf16", "fp16", "bf16-fp32"])
def test_attention_infinities(paged, mode, kv, x):
    """A score of -inf has no weight (fp32 queries: or the head is NaN), NaN and +inf make the head NaN, a V entry its dim."""
    contexts, width = MODES[mode]
    dh, hq, hkv = 64, 8, 2
    cache, table, q, ctx = make(paged, contexts, hq, hkv, dh, 16, kv, x, seed=17)
    q.abs_().clamp_(0.1)
    if width:
        wide = torch.full((len(contexts), width), -1, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        table = wide
    entry = lambda row, pos: (int(table[row, pos // 16]), pos % 16)  # noqa: E731
    hit, rest = slice(4, 8), slice(0, 4)             # query heads of kv head 1 and of kv head 0
    want, want_lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
    check(want, want_lse, q, cache, table, contexts)
    p, at = entry(0, 33)
    kept_k, kept_v = cache.k[p, 1, at].clone(), cache.v[p, 1, at].clone()

    def run():
        out, lse = paged.d3_paged_attention(cache, q, table, ctx, with_lse=True)
        assert torch.equal(out[0, rest], want[0, rest]) and torch.equal(out[1], want[1])
        assert torch.equal(lse[0, rest], want_lse[0, rest]) and torch.equal(lse[1], want_lse[1])
        return out[0, hit], lse[0, hit]

    cache.k[p, 1, at, 7] = -math.inf                 # one position without weight
    out, lse = run()
    if x == FP32 and out.isnan().any():
        assert out.isnan().all(-1).any()
    else:
        cache.k[p, 1, at] = kept_k
        cache.v[p, 1, at] = kept_v
        keep = [i for i in range(contexts[0]) if i != 33]
        ids = table[0].tolist()[: -(-contexts[0] // 16)]
        kd, vd = (torch.stack([t[i].float() for i in ids]).double().permute(1, 0, 2, 3).reshape(hkv, -1, dh)[1:, keep] for t in
                  (cache.k, cache.v))
        close(out[None], lse[None], q[:1, hit], kd, vd, dh ** -0.5, 2.0 ** -16)
    for bad in (math.inf, math.nan):
        cache.k[p, 1, at] = kept_k
        cache.k[p, 1, at, 7] = bad
        out, lse = run()
        assert out.isnan().all() and lse.isnan().all()
    cache.k[p, 1, at] = kept_k
    for bad in (math.inf, -math.inf, math.nan):
        cache.v[p, 1, at] = kept_v
        cache.v[p, 1, at, 7] = bad
        out, lse = run()
        dims = [d for d in range(dh) if d != 7]
        assert not out[:, 7].isfinite().any() and torch.equal(lse, want_lse[0, hit])
        assert torch.equal(out[:, dims], want[0, hit][:, dims])
    cache.v[p, 1, at] = kept_v
    for page in set(table[0].tolist()) - {-1}:       # no position of the head has weight: as a row without context
        cache.k[page, 1, :, 7] = -math.inf
    out, lse = run()
    if x == FP32:
        assert (out.isnan() | (out == 0)).all() and (lse.isnan() | (lse == -math.inf)).all()
    else:
        assert (out == 0).all() and (lse == -math.inf).all()
