"""The constraints on logits behind a loaded model's decode steps: tokens are chosen from the step's own logits and go into the next step."""
import pytest
import torch

from paper_2503_08524_b200 import binding as B
from paper_2503_08524_b200 import block8 as K
from paper_2503_08524_b200 import inputs as I
from test_gpu_block8 import check_logits, logits_form

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 3])
def test_decode_steps_with_constraints(rows):
    shape, dev, seed, plen, steps = I.TINY, "cuda:0", I.BASE_SEED + 5, 9, 6
    V = shape.vocab
    w = I.make_weights(shape, seed, device=dev, gain_jitter=0.1)
    model = B.D3Model(shape, w, rows, 64, rows, start_id=1, kv_fill=B.FILL_COPY, device=dev)
    model.zero_kv()
    history = torch.full((rows, plen + steps + 1), -1, dtype=torch.int32, device=dev)
    for b in range(rows):
        prompt = I.prompt_tokens(shape, seed, b, plen)
        model.d3_prefill(b, prompt.numpy())
        history[b, :plen] = prompt.to(torch.int32).to(dev)
    g = torch.Generator(device=dev).manual_seed(1)
    lengths = torch.full((rows,), plen, dtype=torch.int32, device=dev)
    prompts = lengths.clone()
    masks = torch.randint(-2 ** 31, 2 ** 31, (2, V // 32), generator=g, device=dev).to(torch.int32)
    mask_of = torch.tensor([b % 3 - 1 for b in range(rows)], dtype=torch.int32, device=dev)
    penalties = {k: torch.full((rows,), v, device=dev) for k, v in (("repetition", 1.3), ("frequency", 0.2), ("presence", 0.4))}
    ids = torch.randint(0, V, (rows, 5), generator=g, device=dev).to(torch.int32)
    bias = torch.randn((rows, 5), generator=g, device=dev)
    token = torch.full((rows,), 7, dtype=torch.int32, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    for step in range(steps):
        for b in range(rows):
            history[b, plen + step] = token[b]
        lengths += 1
        logits = model.d3_decode_step(list(range(rows)), None, [step + 1] * rows, 0.9, tokens_dev=token)
        plain, free = K.d3_constrain_logits(logits)
        assert torch.equal(plain, logits) and torch.equal(free, model.d3_argmax(logits))
        kw = dict(history=history, lengths=lengths, prompt=prompts, bias_ids=ids, bias=bias, masks=masks, mask_of=mask_of, **penalties)
        y, dy = logits_form(logits, **kw)
        out, token = K.d3_constrain_logits(logits, out=logits, status=status, **kw)       # in place
        assert out is logits
        check_logits(out, token, y, dy)
        assert int(status) == 0
    model.close()
