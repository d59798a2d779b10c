"""Cases, plain forms and 64-bit values of the 8-bit block operators and of the constraints on logits.

Four operators make up the weight side of a decoder block, and what stands between its logits and a
token, for a caller that runs a block itself:

  norm     the residual sum, the root-mean-square norm and the result in 8 bits with a scale for every
           128 numbers of a row (or in a wider type; or the 8 bits alone, without a norm)
  matmul   rows in 8 bits times a weight matrix in 8 bits that has a scale for each block of 128 x 128
  gated    two such products, silu of one times the other, the result again in 8 bits with scales
  logits   penalties for repeated tokens, biases, a grammar's mask, and the best token that is left

`own` chooses between the plain forms below (elementary torch operations in 32 bits) and the calls that
a user makes of this package.  Sizes are those of the package's own shapes and workloads (7B, 13B and
70B shapes; 1, 4, 8 and 32 rows; prompts) and generic ones beyond them.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1, "none": 0}
BLOCK = 128
E4M3_MAX = 448.0
LEAST = 2.0 ** -100       # a block's largest number counts as this at least, so that its scale is a normal number
EPS = 1e-5


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of the 7B shape, the fp32 residual stream of this package's steps: all latency
        norm("norm 1 row 7B", rows=1, dim=4096, x="fp32", add="fp32", out="e4m3", gain="bf16"),
        # 32 rows of the 13B shape in front of a 16-bit projection
        norm("norm 32 rows 13B bf16", rows=32, dim=5120, x="bf16", add="bf16", out="bf16", gain="bf16"),
        # a prompt at the 70B shape: 16-bit results of a projection onto a 32-bit stream
        norm("norm 8191 rows 70B", rows=8191, dim=8192, x="bf16", add="fp32", out="e4m3", gain="bf16"),
        # what a projection takes that has no norm before it (attention's output, another block's activation)
        norm("quantize 4097 rows fp16", rows=4097, dim=11008, x="fp16", add="none", out="e4m3", gain="none"),
        # one token's queries, keys and values at the 7B shape
        matmul("matmul 1 row 7B", rows=1, k=4096, n=12288, out="bf16"),
        # 32 rows through the 7B shape's down projection: few outputs, long sums
        matmul("matmul 32 rows 7B down", rows=32, k=11008, n=4096, out="bf16"),
        # a few rows at the 70B shape onto the fp32 stream
        matmul("matmul 4 rows 70B fp32", rows=4, k=8192, n=10240, out="fp32"),
        # a prompt at the 70B shape
        matmul("matmul 8191 rows 70B", rows=8191, k=8192, n=8192, out="bf16"),
        # the feed-forward's first half at the 13B shape, 8 rows
        gated("gated 8 rows 13B", rows=8, k=5120, n=13824, out="e4m3"),
        # the same for a prompt at the 7B shape
        gated("gated 2047 rows 7B", rows=2047, k=4096, n=11008, out="e4m3"),
        # one row's choice at this package's vocabulary
        logits("logits 1 row", rows=1, vocab=32000, history=545, prompt=512, biases=5, masks=1, empty=0, x="fp32"),
        # a serving batch over a large vocabulary of odd size, two rows of which a grammar leaves nothing
        logits("logits 250 rows", rows=250, vocab=128001, history=4099, prompt=1024, biases=300, masks=32, empty=2, x="fp32"),
    ]


def norm(name, rows, dim, x, add, out, gain):
    return dict(name=name, op="norm", rows=rows, dim=dim, x=x, add=add, out=out, gain=gain)


def matmul(name, rows, k, n, out):
    return dict(name=name, op="matmul", rows=rows, k=k, n=n, out=out)


def gated(name, rows, k, n, out):
    return dict(name=name, op="gated", rows=rows, k=k, n=n, out=out)


def logits(name, rows, vocab, history, prompt, biases, masks, empty, x):
    return dict(name=name, op="logits", rows=rows, vocab=vocab, history=history, prompt=prompt, biases=biases, masks=masks,
                empty=empty, x=x)


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


WIDTHS = (256, 688, 4096, 5120, 8192, 10240, 11008, 12288, 13824, 28672)


def width(rng, step, top):
    """One of the package's widths, or any multiple of `step`."""
    return rng.choice([w for w in WIDTHS if w <= top] or [step]) if rng.random() < 0.5 else max(step, log_int(rng, step, top) // step * step)


def draw(rng):
    op = rng.choice(("norm", "matmul", "matmul", "gated", "gated", "logits"))
    if op == "norm":
        dim = width(rng, 8, 28672)
        x = rng.choice(("bf16", "fp16", "fp32"))
        gain = rng.choice(("bf16", "fp32", x, "none"))
        c = norm("", log_int(rng, 1, 8191 * 8192 // dim if dim > 4096 else 16384), dim, x, rng.choice(("none", x, "fp32")),
                 "e4m3" if gain == "none" else rng.choice(("e4m3", "e4m3", x, "bf16")), gain)
    elif op == "matmul":
        k = width(rng, 16, 28672)
        n = rng.choice(WIDTHS + (32000,)) if rng.random() < 0.5 else log_int(rng, 1, 32000)
        n = min(n, 8192 * 28672 // k)
        c = matmul("", log_int(rng, 1, min(8191, max(1, 8191 * 8192 * 8192 // (n * k)))), k, n, rng.choice(("bf16", "bf16", "fp16", "fp32")))
    elif op == "gated":
        k = width(rng, 16, 8192)
        n = width(rng, 8, min(28672, 8192 * 28672 // k))
        c = gated("", log_int(rng, 1, min(4096, max(1, 2047 * 4096 * 11008 // (n * k)))), k, n, rng.choice(("e4m3", "e4m3", "bf16", "fp32")))
    else:
        vocab = rng.choice((1024, 32000)) if rng.random() < 0.4 else log_int(rng, 100, 131072)
        rows = log_int(rng, 1, min(512, 250 * 128001 // vocab))
        history = log_int(rng, 1, 8192) if rows < 100 else log_int(rng, 1, 4099)
        c = logits("", rows, vocab, history, rng.randint(0, history), rng.choice((0, 1, log_int(rng, 1, min(300, vocab)))),
                   rng.choice((0, 1, log_int(rng, 1, 64))), rng.choice((0, 0, rows // 4)), rng.choice(("fp32", "fp32", "bf16", "fp16")))
    del c["name"]
    return c


# --------------------------------------------------------------------------------------------- inputs
def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(shape, g, std=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def uniform(shape, g, lo, hi):
    return torch.empty(shape, dtype=torch.float32, device=DEV).uniform_(lo, hi, generator=g)


def blocks(n):
    return -(-n // BLOCK)


def activations(rows, dim, g):
    """What a block's stream looks like: channels of different size, a few of them large."""
    channel = torch.exp(0.5 * normal((dim,), g))
    channel[torch.randint(dim, (max(1, dim // 512),), generator=g, device=DEV)] *= 20.0
    return normal((rows, dim), g) * channel


def rows_in_8_bits(x):
    """(e4m3 [rows][dim], fp32 [rows][blocks])."""
    rows, dim = x.shape
    pad = torch.nn.functional.pad(x, (0, blocks(dim) * BLOCK - dim)).view(rows, -1, BLOCK)
    scale = pad.abs().amax(-1).clamp(min=LEAST) / E4M3_MAX
    q = (pad / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).view(rows, -1)[:, :dim].contiguous().to(torch.float8_e4m3fn)
    return q, scale


def weight_in_8_bits(n, k, g):
    """(e4m3 [n][k], fp32 [blocks of n][blocks of k]): numbers that fill the type's range, scales of their own."""
    q = normal((n, k), g, 100.0).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q, uniform((blocks(n), blocks(k)), g, 0.5, 1.5) * (0.02 / 100.0)


def prepare(case, seed):
    g = generator(seed)
    op = case["op"]
    s = dict(op=op)
    if op == "norm":
        rows, dim, x = case["rows"], case["dim"], TYPES[case["x"]]
        s["x"] = activations(rows, dim, g).to(x)
        s["add"] = None if case["add"] == "none" else (3.0 * activations(rows, dim, g)).to(TYPES[case["add"]])
        s["gain"] = None if case["gain"] == "none" else (1.0 + normal((dim,), g, 0.1)).to(TYPES[case["gain"]])
        s["dtype"] = TYPES[case["out"]]
        if own:
            s["out"] = torch.empty((rows, dim), dtype=s["dtype"], device=DEV)
            s["total"] = None if s["add"] is None else torch.empty_like(s["add"])
            s["scale"] = torch.empty((rows, blocks(dim)), device=DEV) if case["out"] == "e4m3" else None
    elif op in ("matmul", "gated"):
        rows, k, n = case["rows"], case["k"], case["n"]
        s["a"], s["a_scale"] = rows_in_8_bits(activations(rows, k, g))
        s["w"] = [weight_in_8_bits(n, k, g) for _ in range(2 if op == "gated" else 1)]
        s["dtype"] = TYPES[case["out"]]
        if own:
            from paper_2503_08524_b200 import block8
            s["weight"] = [block8.Weight8(q, scale) for q, scale in s["w"]]
            s["out"] = torch.empty((rows, n), dtype=s["dtype"], device=DEV)
            s["scale"] = torch.empty((rows, blocks(n)), device=DEV) if case["out"] == "e4m3" else None
    else:
        rows, vocab, T = case["rows"], case["vocab"], case["history"]
        s["logits"] = normal((rows, vocab), g, 4.0, TYPES[case["x"]])
        # tokens of a text repeat: small numbers are more frequent than large ones
        s["history"] = (uniform((rows, T), g, 0.0, 1.0) ** 3 * vocab).to(torch.int32).clamp_(max=vocab - 1)
        s["lengths"] = torch.randint(T // 2, T + 1, (rows,), generator=g, device=DEV).to(torch.int32)
        s["prompt"] = torch.minimum(s["lengths"], torch.full_like(s["lengths"], case["prompt"]))
        s["repetition"] = uniform((rows,), g, 0.9, 1.5)
        s["frequency"] = uniform((rows,), g, -0.2, 0.5)
        s["presence"] = uniform((rows,), g, -0.2, 0.8)
        s["bias_ids"] = s["bias"] = s["masks"] = s["mask_of"] = None
        if case["biases"]:
            ids = uniform((rows, vocab), g, 0.0, 1.0).topk(min(vocab, case["biases"]), dim=1).indices.to(torch.int32)
            ids[:, 1::7] = -1          # rows have fewer of them than there is room
            s["bias_ids"], s["bias"] = ids.contiguous(), normal(ids.shape, g, 3.0)
        if case["masks"]:
            words = -(-vocab // 32)
            masks = torch.randint(-2 ** 31, 2 ** 31, (case["masks"] + 1, words), generator=g, device=DEV).to(torch.int32)
            masks[-1] = 0              # a state of the grammar that nothing may follow
            s["masks"] = masks
            s["mask_of"] = torch.randint(-1, case["masks"], (rows,), generator=g, device=DEV).to(torch.int32)
            if case["empty"]:
                s["mask_of"][torch.randperm(rows, generator=g, device=DEV)[: case["empty"]]] = case["masks"]
        if own:
            s["out"] = torch.empty_like(s["logits"])
            s["token"] = torch.empty((rows,), dtype=torch.int32, device=DEV)
    return s


# -------------------------------------------------------------------------------------------- one pass
def run(s):
    op = s["op"]
    if own:
        from paper_2503_08524_b200 import block8
        if op == "norm" and s["gain"] is None and s["add"] is None:
            block8.d3_quantize(s["x"], out=s["out"], scale=s["scale"])
            return dict(out=s["out"], scale=s["scale"])
        if op == "norm":
            block8.d3_add_norm(s["x"], s["gain"], add=s["add"], total=s["total"], out=s["out"], scale=s["scale"], eps=EPS)
            return dict(out=s["out"], scale=s["scale"], total=s["total"])
        if op == "matmul":
            block8.d3_matmul8(s["a"], s["a_scale"], s["weight"][0], out=s["out"])
            return dict(out=s["out"])
        if op == "gated":
            block8.d3_gated_matmul8(s["a"], s["a_scale"], s["weight"][0], s["weight"][1], out=s["out"], scale=s["scale"])
            return dict(out=s["out"], scale=s["scale"])
        block8.d3_constrain_logits(s["logits"], history=s["history"], lengths=s["lengths"], prompt=s["prompt"],
                                   repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                                   bias_ids=s["bias_ids"], bias=s["bias"], masks=s["masks"], mask_of=s["mask_of"], out=s["out"],
                                   token=s["token"])
        return dict(out=s["out"], token=s["token"])
    return {"norm": norm_plain, "matmul": matmul_plain, "gated": gated_plain, "logits": logits_plain}[op](s)


def results(y, dtype):
    if dtype == torch.float8_e4m3fn:
        q, scale = rows_in_8_bits(y)
        return dict(out=q, scale=scale)
    return dict(out=y.to(dtype), scale=None)


def norm_plain(s):
    y = s["x"].float()
    total = None
    if s["add"] is not None:
        y = y + s["add"].float()
        total = y.to(s["add"].dtype)
    if s["gain"] is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * s["gain"].float()
    return dict(results(y, s["dtype"]), total=total)


def widened(q, scale, rows_per_scale):
    scale = scale.repeat_interleave(BLOCK, 1)[:, : q.shape[1]]
    return q.float() * scale.repeat_interleave(rows_per_scale, 0)[: q.shape[0]]


def product_plain(s, i):
    return widened(s["a"], s["a_scale"], 1) @ widened(*s["w"][i], BLOCK).T


def matmul_plain(s):
    return dict(out=product_plain(s, 0).to(s["dtype"]))


def gated_plain(s):
    gate, up = product_plain(s, 0), product_plain(s, 1)
    return results(gate / (1.0 + torch.exp(-gate)) * up, s["dtype"])


def logits_plain(s):
    z = s["logits"].float()
    rows, vocab = z.shape
    history, lengths = s["history"].long(), s["lengths"][:, None]
    place = torch.arange(history.shape[1], device=z.device)[None]
    inside = place < lengths
    written = inside & (place >= s["prompt"][:, None])
    seen = torch.zeros((rows, vocab), dtype=torch.int32, device=z.device).scatter_add_(1, history, inside.int())
    count = torch.zeros((rows, vocab), dtype=torch.int32, device=z.device).scatter_add_(1, history, written.int())
    r = s["repetition"][:, None]
    z = torch.where(seen > 0, torch.where(z > 0, z / r, z * r), z)
    z = z - s["frequency"][:, None] * count.float()
    z = z - torch.where(count > 0, s["presence"][:, None], 0.0)
    if s["bias"] is not None:
        there = s["bias_ids"] >= 0
        z = z + torch.zeros_like(z).scatter_add_(1, s["bias_ids"].clamp(min=0).long(), torch.where(there, s["bias"], 0.0))
    if s["masks"] is not None:
        token = torch.arange(vocab, device=z.device)
        bits = (s["masks"][s["mask_of"].clamp(min=0).long()][:, token // 32] >> (token % 32)) & 1
        z = z.masked_fill((bits == 0) & (s["mask_of"] >= 0)[:, None], -math.inf)
    out = z.to(s["logits"].dtype)
    top = out.amax(1, keepdim=True)
    first = torch.where(out == top, torch.arange(vocab, device=z.device), vocab).amin(1)
    return dict(out=out, token=torch.where(top[:, 0] == -math.inf, -1, first).to(torch.int32))


# --------------------------------------------------------------------------------------- 64-bit values
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]

    def in_8_bits(y):
        """What the 8 bits stand for before they are rounded, and the scales."""
        got, scales = torch.empty_like(y), []
        for b in range(0, y.shape[1], BLOCK):
            top = y[:, b:b + BLOCK].abs().max(dim=1).values.clamp(min=LEAST) / E4M3_MAX
            got[:, b:b + BLOCK] = y[:, b:b + BLOCK] / top.unsqueeze(1)
            scales.append(top)
        return dict(out=got, scale=torch.stack(scales, 1))

    def product(q, scale, wq, ws):
        total = torch.zeros((q.shape[0], wq.shape[0]), dtype=torch.float64, device=DEV)
        for b in range(0, q.shape[1], BLOCK):
            part = q[:, b:b + BLOCK].double() @ wq[:, b:b + BLOCK].double().T
            by_row = ws[:, b // BLOCK].double()[torch.arange(wq.shape[0], device=DEV) // BLOCK]
            total += part * scale[:, b // BLOCK].double().unsqueeze(1) * by_row
        return total

    if op == "norm":
        y = s["x"].double()
        total = None
        if s["add"] is not None:
            y = total = y + s["add"].double()
        if s["gain"] is not None:
            y = y / torch.sqrt((y * y).sum(1, keepdim=True) / case["dim"] + EPS) * s["gain"].double()
        return dict(in_8_bits(y) if case["out"] == "e4m3" else dict(out=y, scale=None), total=total)
    if op in ("matmul", "gated"):
        ys = [product(s["a"], s["a_scale"], wq, ws) for wq, ws in s["w"]]
        if op == "matmul":
            return dict(out=ys[0])
        y = ys[0] * torch.sigmoid(ys[0]) * ys[1]
        return in_8_bits(y) if case["out"] == "e4m3" else dict(out=y, scale=None)
    z = s["logits"].double()
    vocab = case["vocab"]
    for b in range(case["rows"]):
        n, p = int(s["lengths"][b]), int(s["prompt"][b])
        used = torch.bincount(s["history"][b, :n].long(), minlength=vocab)
        new = torch.bincount(s["history"][b, p:n].long(), minlength=vocab)
        r = s["repetition"][b].double()
        z[b] = torch.where(used > 0, torch.where(z[b] > 0, z[b] / r, z[b] * r), z[b])
        z[b] -= s["frequency"][b].double() * new + s["presence"][b].double() * (new > 0)
        if s["bias"] is not None:
            ids = s["bias_ids"][b]
            z[b, ids[ids >= 0].long()] += s["bias"][b][ids >= 0].double()
        if s["masks"] is not None and int(s["mask_of"][b]) >= 0:
            words = s["masks"][int(s["mask_of"][b])].cpu().numpy().view("uint8")
            allowed = torch.from_numpy(((words[:, None] >> [0, 1, 2, 3, 4, 5, 6, 7]) & 1).reshape(-1)[:vocab]).to(DEV)
            z[b, allowed == 0] = -math.inf
    return dict(out=z, token=None)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op == "norm":
        rows, dim = case["rows"], case["dim"]
        each = BYTES[case["x"]] + 2 * BYTES[case["add"]] + BYTES[case["out"]]
        return {"bytes": float(rows * dim * each + dim * BYTES[case["gain"]] + (4 * rows * blocks(dim) if case["out"] == "e4m3" else 0)),
                "flops": 6.0 * rows * dim}
    if op in ("matmul", "gated"):
        rows, k, n, mats = case["rows"], case["k"], case["n"], 2 if op == "gated" else 1
        read = rows * k + 4 * rows * blocks(k) + mats * (n * k + 4 * blocks(n) * blocks(k))
        written = rows * n * BYTES[case["out"]] + (4 * rows * blocks(n) if case["out"] == "e4m3" else 0)
        return {"bytes": float(read + written), "flops": 2.0 * mats * rows * n * k}
    rows, vocab = case["rows"], case["vocab"]
    states = min(rows, case["masks"])
    return {"bytes": float(rows * vocab * 2 * BYTES[case["x"]] + 3 * rows * case["history"] + 8 * rows * case["biases"]
                           + 4 * states * -(-vocab // 32) + 24 * rows), "flops": 5.0 * rows * vocab}
