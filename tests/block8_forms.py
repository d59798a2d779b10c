"""The 8-bit block operators in 64 bits, and how far a result may be from them.

A rounding is off by at most half a step: U[type] relative to the value (fp32 2^-24, fp16 2^-11, bf16 2^-8, e4m3 2^-4, there at
least half its smallest number, 2^-10, times the scale)."""
import torch

BLOCK, E4M3_MAX, LEAST = 128, 448.0, 2.0 ** -100
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}
SMALLEST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half of the least number above 0


def blocks(n):
    return -(-n // BLOCK)


def per_block(y):
    """[rows][blocks][128], zeros behind the end."""
    return torch.nn.functional.pad(y, (0, blocks(y.shape[1]) * BLOCK - y.shape[1])).view(y.shape[0], -1, BLOCK)


def widen(scale, n):
    return scale.double().repeat_interleave(BLOCK, 1)[:, :n]


def weight64(q, scale):
    return q.double() * widen(scale, q.shape[1]).repeat_interleave(BLOCK, 0)[: q.shape[0]]


def rows_in_8_bits(x):
    p = per_block(x.float())
    scale = p.abs().amax(-1).clamp(min=LEAST) / E4M3_MAX
    q = (p / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).reshape(x.shape[0], -1)[:, : x.shape[1]]
    return q.to(torch.float8_e4m3fn), scale


def some_rows(rows, k, g, device="cuda"):
    x = torch.randn((rows, k), generator=g, device=device) * torch.exp(0.5 * torch.randn((k,), generator=g, device=device))
    return rows_in_8_bits(x)


def some_weight(n, k, g, device="cuda"):
    q = (torch.randn((n, k), generator=g, device=device) * 100).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q, torch.rand((blocks(n), blocks(k)), generator=g, device=device) * 2e-4 + 1e-4


def product(q, scale, wq, ws):
    """The sums, and how far a kernel's may be off: a block's 128 products, which are whole in 32 bits, are summed with 128 roundings
    (of at most a step of fp32, should the tensor core cut and not round), the scales' product and its product with the sum take
    one rounding each, the blocks' sums one each, and the parts of a cluster 8 more."""
    a, w = q.double() * widen(scale, q.shape[1]), weight64(wq, ws)
    y, size = a @ w.T, a.abs() @ w.abs().T
    return y, size * ((BLOCK + 2 + blocks(q.shape[1]) + 8) * 2.0 ** -23)


def gated(g, dg, u, du):
    """silu(g) u and its error: silu's slope is below 1.1; exp, the sum, the quotient and the product take 2 + 1 + 1 + 1 roundings."""
    s = g * torch.sigmoid(g)
    h = s * u
    return h, 1.1 * dg * (u.abs() + du) + s.abs() * du + h.abs() * 8 * 2.0 ** -24 + 1e-37


def check_wide(got, y, dy):
    near = (y.abs() + dy) * U[got.dtype] + SMALLEST[got.dtype]
    bad = (got.double() - y).abs() > dy + near
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(((got.double() - y).abs() / (dy + near)).max()))


def check_8_bits(q, scale, y, dy):
    """q and scale against numbers in 64 bits that the kernel had with an error of up to dy."""
    n = y.shape[1]
    top, dtop = per_block(y.abs()).amax(-1), per_block(dy).amax(-1)
    want = top.clamp(min=LEAST) / E4M3_MAX
    off = (scale.double() - want).abs()
    assert (off <= dtop / E4M3_MAX + 2 * U[torch.float32] * want).all(), float((off / want).max())
    s = widen(scale, n)
    # the scale's inverse and the product with it: 2 roundings of fp32 in front of the one to 8 bits
    near = (y.abs() + dy) * (U[torch.float8_e4m3fn] * (1 + 2.0 ** -20) + 2.0 ** -22) + s * 2.0 ** -10
    bad = (q.double() * s - y).abs() > dy + near
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


def norm(x, gain, add, eps):
    """(sum, y, error of y) in 64 bits: the sum is rounded once; the squares' sum takes dim / 8 roundings of one thread at most and 14
    in the shuffles, of which the root halves the effect; mean, eps, root, quotient and the two products one each."""
    s = x.double() if add is None else x.double() + add.double()
    if gain is None:
        return s, s, s.abs() * U[torch.float32]
    r = torch.rsqrt((s * s).mean(-1, keepdim=True) + eps)
    y = s * r * gain.double()
    steps = 1 + (min(64, x.shape[1]) + 2 + 14) / 2 + 6
    return s, y, y.abs() * steps * U[torch.float32] + 1e-37
