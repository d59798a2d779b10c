"""Cases, plain forms and 64-bit values of the paged key-value operators.

Three operators make up the cache side of one decode step over many sequences whose lengths live on
the GPU:

  plan       block tables and slot maps from request lengths: pages are taken from and given back to a
             free stack, every new token gets its slot in the pool, its request and its context length
  append     the new tokens' keys (rotated by position) and values go to their slots, the queries are
             rotated next to them
  attention  one new token per row over its pages, split over the cache's length and joined

`own` chooses between the plain forms below (elementary torch operations in 32 bits) and the calls that
a user makes of this package.  Sizes are those of the package's own shapes and workloads (7B, 13B and
70B shapes, 32 rows of 128..1024 positions, 8 rows of 1024, 4 rows of 512) and generic ones beyond them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode step of a few sequences: the call is all latency
        plan("plan 8 decode", requests=8, ctx=(511, 1024), new=(1, 1), release=0, idle=0, page=64),
        # continuous batching: most rows decode, some are new prompts, some finish, some wait
        plan("plan 255 mixed", requests=255, ctx=(0, 8191), new=(1, 97), release=23, idle=17, page=16),
        # a prompt phase: many tokens, few requests
        plan("plan 192 prompts", requests=192, ctx=(0, 33), new=(129, 2048), release=5, idle=3, page=16),
        # 32 rows at the 7B shape, one token each
        append("append 32 rows 7B", tokens=32, per=1, ctx=(128, 1024), hq=32, hkv=32, dh=128, page=64, kv="bf16", x="bf16", layout="head"),
        # prompt tokens at the 70B shape, cache laid out token by token
        append("append 8191 tokens 70B fp16", tokens=8191, per=1170, ctx=(1, 900), hq=64, hkv=8, dh=128, page=32, kv="fp16", x="fp16", layout="token"),
        # prompt tokens at the 13B shape into an 8-bit cache
        append("append 4097 tokens 13B e4m3", tokens=4097, per=513, ctx=(0, 77), hq=40, hkv=40, dh=128, page=16, kv="e4m3", x="bf16", layout="head"),
        # one sequence of the 7B shape right after its 512-token prompt: latency
        attention("attention 1x513 7B", rows=1, ctx=(513, 513), empty=0, hq=32, hkv=32, dh=128, page=64, kv="bf16", q="bf16", layout="head"),
        # the 32-row workload of the 7B shape
        attention("attention 32x1024 7B", rows=32, ctx=(129, 1025), empty=0, hq=32, hkv=32, dh=128, page=64, kv="bf16", q="bf16", layout="head"),
        # four rows at the 70B shape with the activations of this package's steps (fp32)
        attention("attention 4x545 70B fp32", rows=4, ctx=(513, 545), empty=0, hq=64, hkv=8, dh=128, page=32, kv="bf16", q="fp32", layout="head"),
        # one long document: the split over the length is all the parallelism there is
        attention("attention 1x131071 70B fp16", rows=1, ctx=(131071, 131071), empty=0, hq=64, hkv=8, dh=128, page=256, kv="fp16", q="fp16", layout="token"),
        # a full serving batch of ragged lengths, two rows without any context
        attention("attention 64x16384 GQA", rows=64, ctx=(1, 16384), empty=2, hq=32, hkv=8, dh=128, page=16, kv="bf16", q="bf16", layout="token"),
        # the same kind of batch over an 8-bit cache
        attention("attention 96x8192 e4m3", rows=96, ctx=(17, 8192), empty=0, hq=64, hkv=8, dh=128, page=64, kv="e4m3", q="bf16", layout="head"),
    ]


def plan(name, requests, ctx, new, release, idle, page):
    return dict(name=name, op="plan", requests=requests, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1],
                release=release, idle=idle, page=page)


def append(name, tokens, per, ctx, hq, hkv, dh, page, kv, x, layout):
    return dict(name=name, op="append", tokens=tokens, per=per, ctx_lo=ctx[0], ctx_hi=ctx[1], hq=hq, hkv=hkv, dh=dh, page=page,
                kv=kv, x=x, layout=layout)


def attention(name, rows, ctx, empty, hq, hkv, dh, page, kv, q, layout):
    return dict(name=name, op="attention", rows=rows, ctx_lo=ctx[0], ctx_hi=ctx[1], empty=empty, hq=hq, hkv=hkv, dh=dh, page=page,
                kv=kv, q=q, layout=layout)


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


HEADS = ((4, 4), (8, 2), (32, 32), (32, 8), (40, 40), (64, 8), (12, 4), (16, 1), (7, 7), (48, 3))
PAIRS = (("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("e4m3", "bf16"), ("e4m3", "fp16"))


def draw(rng):
    op = rng.choice(("plan", "append", "attention", "attention"))
    page = rng.choice((16, 32, 64, 128, 256))
    if op == "plan":
        requests = log_int(rng, 1, 700)
        new_hi = log_int(rng, 1, max(1, 300000 // requests if requests > 16 else 16384))
        ctx_hi = log_int(rng, 1, 16384)
        c = plan("", requests, (rng.randint(0, ctx_hi), ctx_hi), (rng.randint(0, new_hi), new_hi), rng.randint(0, requests // 4),
                 rng.randint(0, requests // 4), page)
    elif op == "append":
        (hq, hkv), dh, (kv, x) = rng.choice(HEADS), rng.choice((32, 64, 128)), rng.choice(PAIRS)
        tokens = log_int(rng, 1, min(16384, 8191 * 80 * 128 * 2 // ((hq + 2 * hkv) * dh * BYTES[x])))
        ctx_hi = log_int(rng, 1, 3000)
        c = append("", tokens, log_int(rng, 1, tokens), (rng.randint(0, ctx_hi), ctx_hi), hq, hkv, dh, page, kv, x,
                   rng.choice(("head", "token")))
    else:
        (hq, hkv), dh, (kv, q) = rng.choice(HEADS), rng.choice((32, 64, 128)), rng.choice(PAIRS)
        rows = log_int(rng, 1, 300)
        top = 32 * 16384 * 8 * 128 // (rows * hkv * dh) // max(1, hq // hkv // 4)
        ctx_hi = log_int(rng, 1, max(1, min(131072, top)))
        c = attention("", rows, (rng.randint(0, ctx_hi), ctx_hi), rng.choice((0, 0, rows // 8)), hq, hkv, dh, page, kv, q,
                      rng.choice(("head", "token")))
    del c["name"]
    return c


# --------------------------------------------------------------------------------------------- inputs
def spread(n, lo, hi):
    """n lengths evenly over lo..hi: which lengths occur is the case's, which row has which is the seed's."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def ceil_div(a, b):
    return -(-a // b)


def generator(seed, device=None):
    return torch.Generator(device=device or DEV).manual_seed(seed)


def shuffled(values, seed):
    order = torch.randperm(len(values), generator=generator(seed, "cpu"))
    return np.asarray(values, np.int64)[order.numpy()]


def assign(counts, width, n_pages, seed):
    """(table [len(counts)][width] with -1 where there is no page, the pages left over), pages in random order."""
    order = torch.randperm(n_pages, generator=generator(seed, "cpu")).numpy().astype(np.int32)
    table = np.full((len(counts), width), -1, np.int32)
    table[np.arange(width)[None, :] < np.asarray(counts)[:, None]] = order[: int(np.sum(counts))]
    return torch.from_numpy(table).to(DEV), torch.from_numpy(order[int(np.sum(counts)):]).to(DEV)


def normal(shape, dtype, g, std=1.0):
    if dtype == torch.float8_e4m3fn:
        return torch.empty(shape, dtype=torch.float16, device=DEV).normal_(0.0, std, generator=g).clamp_(-E4M3_MAX, E4M3_MAX).to(dtype)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def pool(case, n_pages, g, filled):
    """K and V [page][kv head][position in the page][dim], laid out head by head or token by token; and their scales."""
    shape = (n_pages, case["hkv"], case["page"], case["dh"])
    if case["layout"] == "token":
        shape = (n_pages, case["page"], case["hkv"], case["dh"])
    dtype = TYPES[case["kv"]]
    std = 32.0 if case["kv"] == "e4m3" else 1.0
    kv = [normal(shape, dtype, g, std) if filled else torch.zeros(shape, dtype=torch.float16, device=DEV).to(dtype) for _ in range(2)]
    if case["layout"] == "token":
        kv = [t.permute(0, 2, 1, 3) for t in kv]
    scales = [None, None]
    if case["kv"] == "e4m3":   # one scale per kv head, as a calibration leaves them
        scales = [torch.empty(case["hkv"], device=DEV).uniform_(0.02, 0.05, generator=g) for _ in range(2)]
    return kv[0], kv[1], scales[0], scales[1]


def new_lengths(case):
    """(new tokens of the rows that get some, sum)."""
    n = spread(case["requests"] - case["release"] - case["idle"], case["new_lo"], case["new_hi"])
    return n, sum(n)


def prepare(case, seed):
    g = generator(seed)
    if case["op"] == "plan":
        page, R = case["page"], case["requests"]
        cached = shuffled(spread(R, case["ctx_lo"], case["ctx_hi"]), seed + 1)
        some, total = new_lengths(case)
        new = shuffled(some + [-1] * case["release"] + [0] * case["idle"], seed + 2)
        width = ceil_div(case["ctx_hi"] + case["new_hi"], page) + 1
        have = -(-cached // page)
        n_pages = int(have.sum()) + ceil_div(total, page) + len(some) + 7    # enough however the lengths meet
        table, free = assign(have, width, n_pages, seed + 3)
        stack = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        stack[: free.numel()] = free
        s = dict(op="plan", page=page, max_tokens=total + 5, cached=torch.from_numpy(cached.astype(np.int32)).to(DEV),
                 new=torch.from_numpy(new.astype(np.int32)).to(DEV), table=table, free=stack,
                 n_free=torch.tensor([free.numel()], dtype=torch.int32, device=DEV))
        if own:
            from paper_2503_08524_b200 import paged
            s["plan"] = paged.PagePlan(cached=s["cached"], new_tokens=s["new"], table=table, free=stack, n_free=s["n_free"],
                                       page_size=page, max_tokens=total + 5, cached_out=torch.empty_like(s["cached"]),
                                       n_free_out=torch.empty_like(s["n_free"]))
        return s
    if case["op"] == "append":
        page, T = case["page"], case["tokens"]
        R = ceil_div(T, case["per"])
        cached = shuffled(spread(R, case["ctx_lo"], case["ctx_hi"]), seed + 1)
        row, step = np.arange(T) // case["per"], np.arange(T) % case["per"]
        position = cached[row] + step
        counts = -(-(cached + np.minimum(case["per"], T - np.arange(R) * case["per"])) // page)
        n_pages = int((-(-(cached + case["per"]) // page)).sum()) + 3
        table, _ = assign(counts, int(counts.max()), n_pages, seed + 3)
        slots = table.cpu().numpy()[row, position // page].astype(np.int64) * page + position % page
        pad = 1 + T // 64   # the tail of a call whose size is fixed by a captured graph
        slots = np.concatenate([slots, np.full(pad, -1)])
        position = np.concatenate([position, np.full(pad, -1)])
        N, hq, hkv, dh = T + pad, case["hq"], case["hkv"], case["dh"]
        qkv = normal((N, hq + 2 * hkv, dh), TYPES[case["x"]], g)   # one buffer, as the fused projection leaves it
        k, v, ks, vs = pool(case, n_pages, g, filled=False)
        top = case["ctx_hi"] + case["per"]
        angle = torch.arange(top, device=DEV, dtype=torch.float64)[:, None] * (
            10000.0 ** (-2.0 * torch.arange(dh // 2, device=DEV, dtype=torch.float64) / dh))
        s = dict(op="append", q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], kc=k, vc=v, ks=ks, vs=vs, page=page,
                 slots=torch.from_numpy(slots).to(DEV), context=torch.from_numpy((position + 1).astype(np.int32)).to(DEV),
                 rope=torch.stack([angle.cos(), angle.sin()], -1).float(), q_out=torch.zeros((N, hq, dh), dtype=qkv.dtype, device=DEV))
        if own:
            from paper_2503_08524_b200 import paged
            s["cache"] = paged.PagedKV(k, v, ks, vs)
        return s
    page = case["page"]
    context = shuffled(spread(case["rows"] - case["empty"], case["ctx_lo"], case["ctx_hi"]) + [0] * case["empty"], seed + 1)
    counts = -(-context // page)
    width = max(1, ceil_div(case["ctx_hi"], page))
    n_pages = int(counts.sum()) + 3
    table, _ = assign(counts, width, n_pages, seed + 3)
    k, v, ks, vs = pool(case, n_pages, g, filled=True)
    q = normal((case["rows"], case["hq"], case["dh"]), TYPES[case["q"]], g, 1.5)
    s = dict(op="attention", q=q, kc=k, vc=v, ks=ks, vs=vs, table=table, context=torch.from_numpy(context.astype(np.int32)).to(DEV),
             scale=case["dh"] ** -0.5)
    if own:
        from paper_2503_08524_b200 import paged
        s["cache"] = paged.PagedKV(k, v, ks, vs)
        s["workspace"] = paged.attention_workspace(s["cache"], case["hq"])
    return s


# -------------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        from paper_2503_08524_b200 import paged
        if s["op"] == "plan":
            p = s["plan"]
            p.d3_page_plan()
            return dict(table=s["table"], free=s["free"], n_free=p.n_free_out, cached=p.cached_out, slots=p.slots, row=p.row,
                        context=p.context, first=p.first)
        if s["op"] == "append":
            paged.d3_paged_append(s["cache"], s["k"], s["v"], s["slots"], q=s["q"], q_out=s["q_out"], rope=s["rope"],
                                  context=s["context"])
            return dict(k=s["kc"], v=s["vc"], q=s["q_out"])
        out, lse = paged.d3_paged_attention(s["cache"], s["q"], s["table"], s["context"], scale=s["scale"], workspace=s["workspace"],
                                            with_lse=True)
        return dict(out=out, lse=lse)
    return {"plan": plan_plain, "append": append_plain, "attention": attention_plain}[s["op"]](s)


def plan_plain(s):
    page, table, free = s["page"], s["table"], s["free"]
    cached, new, n_free, T = s["cached"].long(), s["new"].long(), s["n_free"].long(), s["max_tokens"]
    R, W = table.shape
    released, add = new < 0, new.clamp(min=0)
    have = (cached + page - 1) // page
    need = (cached + add + page - 1) // page - have
    column = torch.arange(W, device=table.device)
    back = column < torch.where(released, have, 0)[:, None]
    given = table[back]                                       # row by row, page by page
    stack = torch.arange(given.numel(), device=table.device) + n_free
    free[stack] = given
    top = n_free + given.numel()
    taken = need.cumsum(0) - need
    fresh = (column >= have[:, None]) & (column < (have + need)[:, None])
    rank = taken[:, None] + column - have[:, None]
    table[fresh] = free[top - 1 - rank[fresh]]
    first = torch.cat([add.new_zeros(1), add.cumsum(0)])
    t = torch.arange(T, device=table.device)
    row = torch.searchsorted(first[1:], t, right=True)
    live = row < R
    r = row.clamp(max=R - 1)
    position = torch.where(live, cached[r] + t - first[r], 0)
    slots = table[r, position // page].long() * page + position % page
    return dict(table=table, free=free, n_free=(top - need.sum()).int(), cached=torch.where(released, 0, cached + add).int(),
                slots=torch.where(live, slots, -1), row=torch.where(live, row, -1).int(),
                context=torch.where(live, position + 1, 0).int(), first=first.int())


def rotate(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def to_cache(x, scale, dtype):
    if dtype == torch.float8_e4m3fn:
        return (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype).view(torch.uint8)
    return x.to(dtype)


def append_plain(s):
    live = s["slots"] >= 0
    slots, page = s["slots"][live], s["page"]
    cos, sin = s["rope"][s["context"][live].long() - 1].unbind(-1)
    cos, sin = cos[:, None], sin[:, None]
    for cache, x, scale in ((s["kc"], rotate(s["k"][live], cos, sin), s["ks"]), (s["vc"], s["v"][live].float(), s["vs"])):
        new = to_cache(x, scale, cache.dtype)
        cache.view(new.dtype).permute(0, 2, 1, 3)[slots // page, slots % page] = new
    s["q_out"][live] = rotate(s["q"][live], cos, sin).to(s["q"].dtype)
    return dict(k=s["kc"], v=s["vc"], q=s["q_out"])


def gathered(cache, table, scale):
    """[row][kv head][position][dim] in 32 bits."""
    x = cache.view(torch.uint8)[table].view(cache.dtype) if cache.dtype == torch.float8_e4m3fn else cache[table]
    x = x.permute(0, 2, 1, 3, 4).flatten(2, 3).float()
    return x if scale is None else x * scale[:, None, None]


def attention_plain(s):
    q, context = s["q"], s["context"]
    table = s["table"].long().clamp(min=0)
    B, hq, dh = q.shape
    k = gathered(s["kc"], table, s["ks"])
    hkv, length = k.shape[1], k.shape[2]
    scores = (q.float().reshape(B, hkv, hq // hkv, dh) @ k.transpose(-1, -2)) * s["scale"]
    del k
    inside = torch.arange(length, device=q.device) < context[:, None]
    scores = scores.masked_fill(~inside[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    v = gathered(s["vc"], table, s["vs"]).masked_fill_(~inside[:, None, :, None], 0.0)
    out = (p @ v) / torch.where(total == 0.0, 1.0, total)
    lse = top + torch.log(total)
    return dict(out=out.reshape(B, hq, dh).to(q.dtype), lse=lse.reshape(B, hq))


# --------------------------------------------------------------------------------------- 64-bit values
def exact(case, seed):
    if case["op"] == "plan":
        return None          # whole numbers only
    s = prepare(case, seed)
    if case["op"] == "append":
        keep = [i for i, v in enumerate(s["slots"].tolist()) if v >= 0]
        token = torch.tensor(keep, device=DEV)
        slot = s["slots"][token]
        table = s["rope"][(s["context"][token] - 1).long()].double()
        cos, sin, half = table[..., 0].unsqueeze(1), table[..., 1].unsqueeze(1), case["dh"] // 2

        def turned(x):
            x = x[token].double()
            y = torch.empty_like(x)
            y[..., :half] = x[..., :half] * cos - x[..., half:] * sin
            y[..., half:] = x[..., :half] * sin + x[..., half:] * cos
            return y

        got = {}
        for name, cache, new, scale in (("k", s["kc"], turned(s["k"]), s["ks"]), ("v", s["vc"], s["v"][token].double(), s["vs"])):
            full = torch.zeros(cache.shape, dtype=torch.float64, device=DEV)
            if scale is not None:
                new = (new / scale.double().unsqueeze(1)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).double()
            full[torch.div(slot, case["page"], rounding_mode="floor"), :, slot % case["page"]] = new
            got[name] = full
        got["q"] = torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEV)
        got["q"][token] = turned(s["q"])
        return got
    group = case["hq"] // case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["context"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, : ceil_div(n, case["page"])].tolist()
        for h in range(case["hkv"]):
            k, v = (torch.stack([c[p, h] for p in pages]).double().reshape(-1, case["dh"])[:n] if len(pages) < 64 else
                    c[:, h].view(torch.uint8 if case["kv"] == "e4m3" else c.dtype)[s["table"][b, : len(pages)].long()].view(
                        c.dtype).double().reshape(-1, case["dh"])[:n] for c in (s["kc"], s["vc"]))
            if s["ks"] is not None:
                k, v = k * float(s["ks"][h]), v * float(s["vs"][h])
            z = (s["q"][b, h * group:(h + 1) * group].double() @ k.T) * s["scale"]
            lse[b, h * group:(h + 1) * group] = torch.logsumexp(z, -1)
            out[b, h * group:(h + 1) * group] = torch.softmax(z, -1) @ v
    return dict(out=out, lse=lse)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "plan":
        _, tokens = new_lengths(case)
        R, page = case["requests"], case["page"]
        mean = (case["ctx_lo"] + case["ctx_hi"]) / 2
        moved = case["release"] * mean / page + tokens / page       # pages given back and taken: one id read, one written
        return {"bytes": 4.0 * (3 * R + 1) + 8.0 * moved + 16.0 * (tokens + 5) + 8.0, "flops": 0.0}
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    if case["op"] == "append":
        T, x = case["tokens"], BYTES[case["x"]]
        turned = T * (hq + hkv) * dh
        return {"bytes": float(T * dh * (2 * hq * x + 2 * hkv * (x + BYTES[case["kv"]])) + T * 12 + min(T, case["ctx_hi"] + case["per"]) * dh * 4),
                "flops": 3.0 * turned}
    total = sum(spread(case["rows"] - case["empty"], case["ctx_lo"], case["ctx_hi"]))
    return {"bytes": float(total * hkv * dh * 2 * BYTES[case["kv"]] + case["rows"] * hq * (2 * dh * BYTES[case["q"]] + 4)
                           + 4 * total / case["page"] + 4 * case["rows"]),
            "flops": 4.0 * total * hq * dh}
