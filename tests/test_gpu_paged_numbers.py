"""Attention over a paged cache where its numbers could lose bits or leave the finite range.

Tolerances are those of test_gpu_paged.py (`reference` there), with the term of the weights of two
fp16 numbers, 2^-21, under every 8-bit cache.
"""
import pytest
import torch

from test_gpu_paged import BF16, DEV, E4M3, FP16, make, paged, reference  # noqa: F401  (paged: a fixture)

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
