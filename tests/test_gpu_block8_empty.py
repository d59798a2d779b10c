"""Lists of no entries: a request without a history yet, or without biases, is one of the lengths that the constraints on logits take."""
import pytest
import torch

from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.mark.parametrize("rows,vocab", [(1, 32000), (3, 1001)])
def test_a_history_of_no_entries(rows, vocab):
    z = torch.randn((rows, vocab), generator=torch.Generator(device="cuda").manual_seed(vocab), device="cuda")
    none = torch.empty((rows, 0), dtype=I32, device="cuda")
    whole = torch.zeros(rows, dtype=I32, device="cuda")
    part = torch.full((rows,), 1.3, device="cuda")
    companions = dict(lengths=whole, prompt=whole, repetition=part, frequency=part, presence=part)
    some = [dict(), companions] + [{k: v} for k, v in companions.items()]
    for kw in some:
        status = torch.zeros(1, dtype=I32, device="cuda")
        out, token = K.d3_constrain_logits(z, history=none, status=status, **kw)
        assert torch.equal(out, z) and torch.equal(token, z.argmax(1).to(I32)) and int(status) == 0
    status = torch.zeros(1, dtype=I32, device="cuda")
    out, _ = K.d3_constrain_logits(z, bias_ids=none, bias=torch.empty((rows, 0), device="cuda"), status=status)
    assert torch.equal(out, z) and int(status) == 0


@pytest.mark.parametrize("name", ["lengths", "prompt"])
@pytest.mark.parametrize("value", [1, -1])
def test_lengths_of_a_history_of_no_entries_are_checked(name, value):
    z = torch.randn((4, 300), device="cuda")
    bad = torch.zeros(4, dtype=I32, device="cuda")
    bad[2] = value
    status = torch.zeros(1, dtype=I32, device="cuda")
    out, _ = K.d3_constrain_logits(z, history=torch.empty((4, 0), dtype=I32, device="cuda"), status=status, **{name: bad})
    assert torch.equal(out, z) and int(status) == B.EINVAL
