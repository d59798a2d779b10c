"""8-bit block operators on the GPU against 64-bit forms (block8_forms.py)."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import block8 as K

pytestmark = pytest.mark.gpu
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


def gen(seed=1):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(rows, width, dtype, extra, fill=7.0):
    """A matrix whose rows lie `extra` numbers further apart, inside a buffer with rows of its own behind it."""
    buf = torch.full((rows + 2, width + extra), fill, device="cuda").to(dtype)
    return buf, buf[:rows, :width]


# ------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("rows,dim", [(1, 8), (1, 4096), (3, 120), (5, 128), (7, 136), (33, 256), (601, 248), (2, 688), (4, 8192), (700, 1032),
                                      (593, 5120), (2, 11008), (3, 28672), (1, 65536)])
@pytest.mark.parametrize("x,add,gain,out", [(FP32, FP32, BF16, E4M3), (BF16, FP32, BF16, E4M3), (BF16, None, BF16, BF16), (FP16, FP16, FP32, FP16),
                                            (FP32, None, FP16, FP32), (BF16, BF16, None, E4M3), (FP16, None, None, E4M3)])
def test_norm(rows, dim, x, add, gain, out):
    g = gen(rows * dim)
    channel = torch.exp(torch.randn((dim,), generator=g, device="cuda"))
    xs = (torch.randn((rows, dim), generator=g, device="cuda") * channel).to(x)
    ad = None if add is None else (3 * torch.randn((rows, dim), generator=g, device="cuda") * channel).to(add)
    ga = None if gain is None else (1 + 0.1 * torch.randn((dim,), generator=g, device="cuda")).to(gain)
    o, sc, total = K.d3_add_norm(xs, ga, add=ad, dtype=out, eps=1e-5)
    s, y, dy = F.norm(xs, ga, ad, 1e-5)
    if add is None:
        assert total is None
    else:
        F.check_wide(total, s, s.abs() * F.U[FP32])
    if out is E4M3:
        F.check_8_bits(o, sc, y, dy)
    else:
        assert sc is None
        F.check_wide(o, y, dy)


def test_norm_leaves_what_is_beside_its_rows_and_works_in_place():
    g = gen()
    x = torch.randn((9, 264), generator=g, device="cuda").to(BF16)
    bx, vx = strided(9, 264, BF16, 24)
    vx.copy_(x)
    stream = torch.randn((9, 264), generator=g, device="cuda")
    bs, vs = strided(9, 264, FP32, 8)
    vs.copy_(stream)
    bo, vo = strided(9, 264, torch.uint8, 8)
    bc, vc = strided(9, 3, FP32, 5)
    gain = torch.rand((264,), generator=g, device="cuda")
    o, sc, total = K.d3_add_norm(vx, gain, add=vs, total=vs, out=vo.view(E4M3), scale=vc)
    s, y, dy = F.norm(x, gain, stream, 1e-5)
    F.check_wide(vs, s, s.abs() * F.U[FP32])
    F.check_8_bits(vo.view(E4M3), vc, y, dy)
    assert total is vs and sc is vc
    for buf, view in ((bs, vs), (bo, vo), (bc, vc)):
        rest = buf.clone()
        rest[: view.shape[0], : view.shape[1]] = 7
        assert (rest == 7).all()
    # the result on x itself
    y2 = x.clone()
    K.d3_add_norm(y2, gain, out=y2)
    _, want, dw = F.norm(x, gain, None, 1e-5)
    F.check_wide(y2, want, dw)


def test_norm_of_zeros_small_numbers_and_what_is_not_finite():
    x = torch.zeros((5, 384), device="cuda")
    x[1] = 1e-30                      # below 2^-100 times 448 a block keeps its zeros
    x[2, 5] = float("nan")
    x[3, 130] = float("inf")
    x[4, 300] = 3.0
    q, s = K.d3_quantize(x)
    assert (q[0].double() == 0).all() and (s[0] == 2.0 ** -100 / 448).all()
    F.check_8_bits(q[1:2], s[1:2], x[1:2].double(), torch.zeros_like(x[1:2], dtype=torch.float64))
    assert torch.isnan(s[2]).tolist() == [True, False, False] and torch.isinf(s[3]).tolist() == [False, True, False]
    v = q.double() * F.widen(s, 384)
    assert torch.isnan(v[2, :128]).all() and (v[2, 128:] == 0).all()
    assert torch.isnan(v[3, 128:256]).all() and (v[3, :128] == 0).all()
    # 448 times a scale of 3 / 448 that was rounded once to fp32
    assert abs(float(v[4, 300]) - 3.0) <= 3.0 * 2.0 ** -24 and (v[4] != 0).sum() == 1
    ones = torch.ones((384,), device="cuda")
    o, sc, _ = K.d3_add_norm(x, ones, eps=0.0)      # 0 / 0
    assert torch.isnan(sc[0]).all() and torch.isnan(o[0].float()).all()
    o, sc, _ = K.d3_add_norm(x, ones)
    assert (o[0].float() == 0).all()


def test_norm_of_a_broadcast_row():
    g = gen()
    x = torch.randn((1, 512), generator=g, device="cuda").expand(6, 512)
    add = torch.randn((6, 512), generator=g, device="cuda")
    gain = torch.ones((512,), device="cuda")
    o, _, total = K.d3_add_norm(x, gain, add=add, dtype=FP32)
    s, y, dy = F.norm(x, gain, add, 1e-5)
    F.check_wide(total, s, s.abs() * F.U[FP32])
    F.check_wide(o, y, dy)


# -------------------------------------------------------------------------------------------- weights
@pytest.mark.parametrize("n,k,dtype", [(1, 16, FP32), (127, 688, BF16), (128, 128, FP16), (300, 1040, BF16), (4096, 256, FP32)])
def test_quantized_weights(n, k, dtype):
    g = gen(n)
    w = (0.02 * torch.randn((n, k + 8), generator=g, device="cuda")).to(dtype)[:, :k]
    w8 = K.d3_quantize_weight(w)
    q = torch.nn.functional.pad(w.double().abs(), (0, F.blocks(k) * 128 - k, 0, F.blocks(n) * 128 - n))
    top = q.view(F.blocks(n), 128, F.blocks(k), 128).amax((1, 3))
    assert ((w8.scale.double() - top / 448).abs() <= 2 * 2.0 ** -24 * top / 448).all()
    s = F.widen(w8.scale, k).repeat_interleave(128, 0)[:n]
    assert ((F.weight64(w8.q, w8.scale) - w.double()).abs() <= w.double().abs() * (2.0 ** -4 * (1 + 2.0 ** -20) + 2.0 ** -22) + s * 2.0 ** -10).all()
    again = K.d3_quantize_weight(2 * w, out=w8)
    assert again is w8 and ((w8.scale.double() - 2 * top / 448).abs() <= 4 * 2.0 ** -24 * top / 448).all()


# -------------------------------------------------------------------------------------------- products
SHAPES = [(1, 16, 1), (1, 4096, 12288), (2, 112, 127), (15, 688, 256), (16, 128, 128), (17, 144, 129), (31, 1024, 1000), (32, 11008, 4096),
          (33, 256, 257), (64, 5120, 640), (65, 688, 688), (100, 4096, 384), (127, 272, 100), (128, 2048, 4096), (129, 128, 128), (200, 4096, 1000),
          (257, 688, 3), (300, 1040, 1300), (1000, 512, 2000), (2047, 4096, 520)]


@pytest.mark.parametrize("rows,k,n", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
def test_matmul(rows, k, n, dtype):
    g = gen(rows + k + n)
    a, s = F.some_rows(rows, k, g)
    wq, ws = F.some_weight(n, k, g)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = K.d3_matmul8(a, s, K.Weight8(wq, ws), dtype=dtype, status=status)
    y, dy = F.product(a, s, wq, ws)
    F.check_wide(out, y, dy)
    assert int(status) == 0


@pytest.mark.parametrize("rows,k,n", SHAPES)
@pytest.mark.parametrize("dtype", [E4M3, BF16, FP32])
def test_gated(rows, k, n, dtype):
    g = gen(rows + k + n)
    a, s = F.some_rows(rows, k, g)
    gate, up = F.some_weight(n, k, g), F.some_weight(n, k, g)
    out, scale = K.d3_gated_matmul8(a, s, K.Weight8(*gate), K.Weight8(*up), dtype=dtype)
    h, dh = F.gated(*F.product(a, s, *gate), *F.product(a, s, *up))
    if dtype is E4M3:
        F.check_8_bits(out, scale, h, dh)
    else:
        assert scale is None
        F.check_wide(out, h, dh)


@pytest.mark.parametrize("rows", [1, 30, 120, 140, 400])
@pytest.mark.parametrize("extra", [1, 3, 4, 16])
def test_products_between_strides(rows, extra):
    k, n = 400, 333
    g = gen(rows)
    a, s = F.some_rows(rows, k, g)
    ba, va = strided(rows, k, torch.uint8, 48)
    va.copy_(a.view(torch.uint8))
    bs, vs = strided(rows, F.blocks(k), FP32, 3)
    vs.copy_(s)
    weights = []
    for i in range(2):
        wq, ws = F.some_weight(n, k, g)
        bw, vw = strided(n, k, torch.uint8, 16)
        vw.copy_(wq.view(torch.uint8))
        weights.append(K.Weight8(vw.view(E4M3), ws))
    args = (va.view(E4M3), vs)
    y, dy = F.product(a, s, weights[0].q, weights[0].scale)
    h, dh = F.gated(y, dy, *F.product(a, s, weights[1].q, weights[1].scale))
    bo, vo = strided(rows, n, BF16, extra)
    K.d3_matmul8(*args, weights[0], out=vo)
    F.check_wide(vo, y, dy)
    b8, v8 = strided(rows, n, torch.uint8, extra)
    bc, vc = strided(rows, F.blocks(n), FP32, extra)
    K.d3_gated_matmul8(*args, *weights, out=v8.view(E4M3), scale=vc)
    F.check_8_bits(v8.view(E4M3), vc, h, dh)
    for buf, view in ((bo, vo), (b8, v8), (bc, vc)):
        rest = buf.clone()
        rest[: view.shape[0], : view.shape[1]] = 7
        assert (rest == 7).all()


@pytest.mark.parametrize("rows", [3, 130])
def test_rows_that_are_not_finite_stay_by_themselves(rows):
    k, n = 512, 384
    g = gen()
    a, s = F.some_rows(rows, k, g)
    w = F.some_weight(n, k, g)
    y, dy = F.product(a, s, *w)
    s = s.clone()
    s[0, 1], s[2, 3] = float("nan"), float("inf")
    a.view(torch.uint8)[1, 5] = 0x7f           # a NaN
    out = K.d3_matmul8(a, s, K.Weight8(*w), dtype=FP32)
    assert torch.isnan(out[0]).all() and torch.isnan(out[1]).all() and not torch.isfinite(out[2]).any()
    F.check_wide(out[3:], y[3:], dy[3:])


@pytest.mark.parametrize("rows", [1, 40, 128, 129, 700])
def test_the_same_call_gives_the_same_bits(rows):
    g = gen()
    a, s = F.some_rows(rows, 4096, g)
    w = K.Weight8(*F.some_weight(4096, 4096, g))
    first = K.d3_matmul8(a, s, w, dtype=FP32)
    for _ in range(5):
        assert torch.equal(K.d3_matmul8(a, s, w, dtype=FP32), first)


def test_no_rows():
    w = K.Weight8(*F.some_weight(200, 256, gen()))
    a, s = torch.empty((0, 256), dtype=E4M3, device="cuda"), torch.empty((0, 2), device="cuda")
    assert K.d3_matmul8(a, s, w).shape == (0, 200)
    out, scale = K.d3_gated_matmul8(a, s, w, w)
    assert out.shape == (0, 200) and scale.shape == (0, 2)
    o, sc, t = K.d3_add_norm(torch.empty((0, 256), device="cuda"), None, add=torch.empty((0, 256), device="cuda"))
    assert o.shape == (0, 256) and sc.shape == (0, 2) and t.shape == (0, 256)


# -------------------------------------------------------------------------------------------- logits
def logits_form(z, history=None, lengths=None, prompt=None, repetition=None, frequency=None, presence=None, bias_ids=None, bias=None, masks=None,
                mask_of=None):
    """Row by row in 64 bits: (values, how far fp32 may be off: a rounding for each of six steps (1 / repetition is one), of
    the numbers that take part)."""
    y = z.double().cpu().clone()
    size = y.abs()
    rows, vocab = y.shape
    for b in range(rows):
        if history is not None:
            ids = history[b].tolist()
            n = len(ids) if lengths is None else min(max(int(lengths[b]), 0), len(ids))
            p = 0 if prompt is None else min(max(int(prompt[b]), 0), len(ids))
            count = {}
            for i, t in enumerate(ids[:n]):
                if 0 <= t < vocab:
                    count[t] = count.get(t, 0) + (i >= p)
            r = 1.0 if repetition is None else float(repetition[b])
            for t, c in count.items():
                v = float(y[b, t])
                v = v / r if v > 0 else v * r
                size[b, t] = abs(v)
                if c:
                    f, q = (0.0 if frequency is None else float(frequency[b])), (0.0 if presence is None else float(presence[b]))
                    size[b, t] += abs(f * c) + abs(q)
                    v -= f * c + q
                y[b, t] = v
        if bias_ids is not None:
            for t, v in dict(zip(bias_ids[b].tolist(), bias[b].tolist())).items():     # (the last one of an id)
                if 0 <= t < vocab:
                    y[b, t] += v
                    size[b, t] += abs(v)
        if mask_of is not None and 0 <= int(mask_of[b]) < masks.shape[0]:
            words = masks[int(mask_of[b])].tolist()
            for t in range(vocab):
                if not (words[t // 32] >> (t % 32)) & 1:
                    y[b, t] = float("-inf")
    return y, size * 6 * 2.0 ** -24


def check_logits(out, token, y, dy):
    got = out.double().cpu()
    gone = torch.isinf(y) & (y < 0)
    assert torch.equal(torch.isinf(got) & (got < 0), gone)
    near = dy + (y.abs() + dy) * F.U[out.dtype] + F.SMALLEST[out.dtype]
    assert ((got - y).abs()[~gone] <= near[~gone]).all()
    for b in range(out.shape[0]):
        v = out[b].float()
        top = v[~torch.isnan(v)].max() if (~torch.isnan(v)).any() else torch.tensor(float("-inf"))
        want = -1 if float(top) == float("-inf") else int((v == top).nonzero()[0])
        assert int(token[b]) == want, b


def some_logits(rows, vocab, n, m, states, dtype, seed):
    g = gen(seed)

    def rand(*shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo
    z = (4 * torch.randn((rows, vocab), generator=g, device="cuda")).to(dtype)
    history = (rand(rows, n) ** 2 * vocab).to(torch.int32).clamp(max=vocab - 1) if n else None
    lengths = torch.randint(0, n + 1, (rows,), generator=g, device="cuda").to(torch.int32)
    kw = {} if not n else dict(history=history, lengths=lengths, prompt=lengths // 2, repetition=rand(rows, lo=0.8, hi=1.5),
                               frequency=rand(rows, lo=-0.3, hi=0.3), presence=rand(rows, lo=-0.5, hi=0.5))
    if m:
        ids = torch.randint(-1, vocab, (rows, m), generator=g, device="cuda").to(torch.int32)     # some twice
        kw.update(bias_ids=ids, bias=torch.randn((rows, m), generator=g, device="cuda"))
    if states:
        masks = torch.randint(-2 ** 31, 2 ** 31, (states, -(-vocab // 32)), generator=g, device="cuda").to(torch.int32)
        masks[states - 1] = 0
        kw.update(masks=masks, mask_of=torch.randint(-1, states, (rows,), generator=g, device="cuda").to(torch.int32))
    return z, kw


@pytest.mark.parametrize("rows,vocab,n,m,states,dtype", [
    (1, 1, 3, 1, 1, FP32), (1, 31, 0, 0, 2, FP32), (2, 33, 5, 0, 0, BF16), (3, 1000, 50, 7, 3, FP32), (5, 1024, 1, 1, 0, FP16), (2, 2047, 300, 0, 4, FP32),
    (4, 4099, 2000, 64, 2, BF16), (1, 32000, 545, 5, 1, FP32), (3, 32003, 4000, 300, 3, FP32), (2, 70001, 100, 3, 2, FP16)])
def test_logits(rows, vocab, n, m, states, dtype):
    z, kw = some_logits(rows, vocab, n, m, states, dtype, vocab + n)
    y, dy = logits_form(z, **kw)
    out, token = K.d3_constrain_logits(z, **kw)
    check_logits(out, token, y, dy)
    for extra in (8, 1, 3):                  # in place, and from rows that start anywhere to rows that start elsewhere
        buf, view = strided(rows, vocab, dtype, extra)
        view.copy_(z)
        other, there = (buf, view) if extra != 3 else strided(rows, vocab, dtype, 6)
        out2, token2 = K.d3_constrain_logits(view, out=there, **kw)
        assert torch.equal(there, out) and torch.equal(token, token2)
        rest = other.clone()
        rest[:rows, :vocab] = 7
        assert (rest == 7).all()


@pytest.mark.parametrize("n,m", [(32767, 3), (32768, 3), (5, 65535), (5, 65536), (70000, 70000)])
def test_logits_with_long_lists(n, m):
    z, kw = some_logits(2, 9000, n, m, 2, FP32, n + m)
    kw["history"][1] = 17                    # one token, as often as the row is long
    kw["lengths"][:] = n
    kw["prompt"][:] = torch.tensor([n // 2, 0], dtype=torch.int32)
    y, dy = logits_form(z, **kw)
    check_logits(*K.d3_constrain_logits(z, **kw), y, dy)


def test_logits_that_are_not_numbers_and_ties():
    z = torch.zeros((6, 40000), device="cuda")
    z[0, 7] = float("nan")
    z[1] = float("nan")
    z[2] = float("-inf")
    z[3, 39999] = float("inf")
    z[4, [39000, 20000, 39001]] = 2.0
    masks = torch.full((2, 1250), -1, dtype=torch.int32, device="cuda")
    masks[0, 0] = ~(1 << 7)                         # what is masked may be a NaN
    masks[1] = 0
    mask_of = torch.tensor([0, -1, -1, -1, -1, 1], dtype=torch.int32, device="cuda")
    out, token = K.d3_constrain_logits(z, masks=masks, mask_of=mask_of)
    assert token.tolist() == [0, -1, -1, 39999, 20000, -1]
    assert float(out[0, 7]) == float("-inf") and torch.isnan(out[1]).all()


@pytest.mark.parametrize("rows,vocab", [(1, 32000), (300, 1000)])
def test_logits_without_a_token(rows, vocab):
    """The C ABI's form that wants no token, and parts that are left out one by one."""
    import ctypes as C
    z, kw = some_logits(rows, vocab, 40, 3, 2, FP32, vocab)
    out = torch.zeros_like(z)
    args = K.ConstrainLogitsArgs(C.sizeof(K.ConstrainLogitsArgs), 2, rows, vocab, 0, 0, 0, z.data_ptr(), out.data_ptr(), vocab, vocab, 0, 0, 0)
    assert K.LIB.d3_constrain_logits(C.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, z)
    for left in (("history", "lengths", "prompt", "repetition", "frequency", "presence"), ("lengths",), ("prompt", "repetition"), ("frequency",), ("presence",),
                 ("bias_ids", "bias"), ("masks", "mask_of")):
        some = {k: v for k, v in kw.items() if k not in left}
        check_logits(*K.d3_constrain_logits(z, **some), *logits_form(z, **some))


def test_logits_report_bad_entries_and_go_on():
    z, kw = some_logits(4, 3000, 20, 6, 2, FP32, 5)
    for name, at, value in (("history", (1, 0), 3000), ("lengths", 2, 21), ("lengths", 2, -1), ("prompt", 0, 99), ("bias_ids", (3, 2), 1 << 30),
                            ("mask_of", 1, 2), (None, None, None)):
        bad = {k: v.clone() for k, v in kw.items()}
        bad["lengths"][1] = 20
        if name:
            bad[name][at] = value
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, token = K.d3_constrain_logits(z, status=status, **bad)
        y, dy = logits_form(z, **bad)
        check_logits(out, token, y, dy)
        assert int(status) == (-1 if name else 0), name


# the ways a product can take (rows of a CTA, k cut between CTAs, either kernel), whatever the sizes that choose them
@pytest.mark.parametrize("rows,k,n", [(1, 28672, 16), (20, 4096, 256), (40, 11008, 130), (100, 2064, 1000), (128, 8192, 1024), (256, 8192, 1024), (300, 8192, 500),
                                      (1000, 4096, 260), (3000, 1040, 200), (257, 4096, 2304), (520, 272, 3000)])
def test_products_of_middling_sizes(rows, k, n):
    g = gen(rows + k + n)
    a, s = F.some_rows(rows, k, g)
    gate, up = F.some_weight(n, k, g), F.some_weight(n, k, g)
    y, dy = F.product(a, s, *gate)
    F.check_wide(K.d3_matmul8(a, s, K.Weight8(*gate), dtype=FP32), y, dy)
    h, dh = F.gated(y, dy, *F.product(a, s, *up))
    F.check_8_bits(*K.d3_gated_matmul8(a, s, K.Weight8(*gate), K.Weight8(*up)), h, dh)
