"""The repetition penalty divides: what fp32 division gives, to the bit, for any penalty."""
import pytest
import torch

from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16])
@pytest.mark.parametrize("vocab,two", [(3001, False), (3001, True), (40000, False)])
def test_a_repetition_penalty_divides(dtype, vocab, two):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows, n = 6, 40000 if two else 2000
    z = (4 * torch.randn((rows, vocab), generator=g, device="cuda")).to(dtype)
    history = torch.randint(0, vocab // 2, (rows, n), generator=g, device="cuda").to(torch.int32)
    r = torch.tensor([1.1, 1.3, 0.7, 3.0, 1.0, 1e-3], device="cuda")
    out, _ = K.d3_constrain_logits(z, history=history, repetition=r)
    seen = torch.zeros((rows, vocab), dtype=torch.bool).scatter_(1, history.long().cpu(), True)
    v, by = z.float().cpu(), r.cpu()[:, None]
    assert seen.any() and not seen.all()
    assert torch.equal(out.cpu(), torch.where(seen, torch.where(v > 0, v / by, v * by), v).to(dtype))


def test_a_penalty_whose_reciprocal_is_infinite():
    z = torch.full((2, 500), 1e-10, device="cuda")
    z[:, 3] = 1e-30
    history = torch.tensor([[3, 499], [3, 7]], dtype=torch.int32, device="cuda")
    r = torch.tensor([2e-39, 1e-39], device="cuda")                    # 1 / r is above the largest number, z / r is not
    out, token = K.d3_constrain_logits(z, history=history, repetition=r)
    want = z.cpu().clone()
    for b in range(2):
        for t in history[b].tolist():
            want[b, t] = z.cpu()[b, t] / r.cpu()[b]
    assert torch.isfinite(want).all() and torch.equal(out.cpu(), want) and token.tolist() == [499, 7]
