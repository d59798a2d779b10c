"""The 8 bits of a number are those of its quotient by the block's scale, as fp32 division gives it: nothing of them is left to a tolerance
where the inputs themselves are quantised."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


def codes(x, scale):
    """The quotients in 8 bits, on the CPU (whose division is IEEE's): scale [rows][blocks]."""
    p = F.per_block(x.float().cpu()) / scale.cpu()[..., None]
    return p.clamp(-448.0, 448.0).reshape(x.shape[0], -1)[:, : x.shape[1]].to(E4M3).view(torch.uint8)


def numbers(kind, rows, dim, dtype, seed):
    """Kinds of rows: `ties`, whole multiples of a power of two in blocks whose scale is one, so that many lie in the middle between two
    codes; `near`, middles between codes times the scale, rounded, and the numbers next to them; and numbers of any size."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "ties":
        x = torch.randint(-447, 448, (rows, dim), generator=g, device="cuda").float()
        x[:, ::128] = 448.0
        x[:, 1::128] = -0.0
        step = torch.randint(-6, 6, (rows, 1), generator=g, device="cuda").float()
        return (x * 2.0 ** step).to(dtype)
    if kind in ("near", "near tiny"):
        top = 1.0 + torch.rand((rows, 1), generator=g, device="cuda")
        if kind == "near tiny":                  # (the remainders of such a division are below the smallest number)
            top = top * 2.0 ** -98
        middle = (2 * torch.randint(8, 16, (rows, dim), generator=g, device="cuda") + 1) * 2.0 ** torch.randint(-4, 5, (rows, dim), generator=g, device="cuda")
        x = middle * (top.to(dtype).float() / 448.0)
        x = x + x * 2.0 ** -24 * torch.randint(-2, 3, (rows, dim), generator=g, device="cuda")
        x[:, ::128] = top
        return x.to(dtype)
    size = {"ordinary": 1.0, "tiny": 2.0 ** -95, "subnormal": 2.0 ** -135, "large": 2.0 ** 120}[kind]
    channel = torch.exp(2 * torch.randn((dim,), generator=g, device="cuda")).clamp(max=16.0)
    return (torch.randn((rows, dim), generator=g, device="cuda") * channel * size).to(dtype)


KINDS = [(k, t) for t in (FP32, BF16) for k in ("ties", "near", "near tiny", "ordinary", "tiny", "subnormal", "large")] + [(k, FP16) for k in ("ties", "near", "ordinary")]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("rows,dim", [(1, 136), (300, 4096), (2000, 248)])
def test_codes_of_rows(kind, dtype, rows, dim):
    x = numbers(kind, rows, dim, dtype, rows + dim)
    q, s = K.d3_quantize(x)
    assert torch.equal(s.cpu(), F.per_block(x.float().cpu()).abs().amax(-1).clamp(min=F.LEAST) / 448.0)
    assert torch.equal(q.view(torch.uint8).cpu(), codes(x, s))
    q2, s2, _ = K.d3_add_norm(x, None, add=torch.zeros_like(x))     # the other kernel; x + 0 loses the sign of -0 alone
    assert torch.equal(s2, s) and torch.equal(q2.float(), q.float())


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_codes_of_weights(kind, dtype):
    n, k = 300, 656
    w = numbers(kind, n, k, dtype, 7)
    w8 = K.d3_quantize_weight(w)
    by_row = w8.scale.repeat_interleave(128, 0)[:n]
    assert torch.equal(w8.q.view(torch.uint8).cpu(), codes(w, by_row))


def test_codes_of_blocks_that_are_not_finite():
    """Beside an infinity the finite numbers are zeros (of an infinite scale), beside a NaN all are NaN."""
    x = torch.ones((2, 256), device="cuda")
    x[0, 3], x[1, 130] = float("inf"), float("nan")
    q, s = K.d3_quantize(x)
    assert torch.isinf(s[0, 0]) and torch.isnan(s[1, 1])
    v = q.float()
    assert torch.isnan(v[0, 3]) and (v[0, [i for i in range(128) if i != 3]] == 0).all() and torch.isnan(v[1, 128:]).all()
    assert (v[0, 128:] == 448).all() and (v[1, :128] == 448).all()
