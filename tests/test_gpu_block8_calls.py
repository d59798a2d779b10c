"""Calls of the 8-bit block operators: a decoder block of them with the paged ones, eager and captured; streams, other callers' buffers,
in-place marks."""
import pytest
import torch

import block8_forms as F
from paper_2503_08524_b200 import block8 as K
from paper_2503_08524_b200 import paged as P

pytestmark = pytest.mark.gpu
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn

D, HQ, HKV, DH, FF, V = 512, 4, 2, 64, 688, 1024


class Block:
    """One decoder block and the head in 8 bits, as a caller that runs a block itself would keep it: weights quantised once, a pool of pages,
    buffers of the step's size."""

    def __init__(self, rows, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(n, k):
            return K.d3_quantize_weight((0.05 * torch.randn((n, k), generator=g, device="cuda")).to(BF16))
        self.g, self.rows = g, rows
        self.wqkv, self.wo, self.gate, self.up, self.down, self.head = w((HQ + 2 * HKV) * DH, D), w(D, HQ * DH), w(FF, D), w(FF, D), w(D, FF), w(V, D)
        self.norm1, self.norm2, self.norm3 = ((1 + 0.1 * torch.randn((D,), generator=g, device="cuda")).to(BF16) for _ in range(3))
        pages, page = 4 * rows + 1, 16
        self.cache = P.PagedKV(torch.zeros((pages, HKV, page, DH), dtype=BF16, device="cuda"), torch.zeros((pages, HKV, page, DH), dtype=BF16, device="cuda"))
        self.plan = P.PagePlan(cached=torch.zeros(rows, dtype=torch.int32, device="cuda"), new_tokens=torch.ones(rows, dtype=torch.int32, device="cuda"),
                               table=torch.full((rows, 4), -1, dtype=torch.int32, device="cuda"), free=torch.arange(pages, dtype=torch.int32, device="cuda"),
                               n_free=torch.tensor([pages], dtype=torch.int32, device="cuda"), page_size=page, max_tokens=rows)
        self.rope = P.d3_rope_table(64, DH)
        self.workspace = P.attention_workspace(self.cache, HQ)
        self.x = torch.zeros((rows, D), device="cuda")
        self.history = torch.full((rows, 64), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.repetition = torch.full((rows,), 1.2, device="cuda")
        self.masks = torch.randint(-2 ** 31, 2 ** 31, (2, V // 32), generator=g, device="cuda").to(torch.int32)
        self.mask_of = torch.tensor([b % 3 - 1 for b in range(rows)], dtype=torch.int32, device="cuda")
        self.embed = torch.randn((V, D), generator=g, device="cuda")

    def step(self):
        """x goes through the block and the head; every tensor on the way, by name."""
        s = {"x": self.x}
        self.plan.d3_page_plan()
        s["h1"], s["h1s"], _ = K.d3_add_norm(self.x, self.norm1)
        s["qkv"] = K.d3_matmul8(s["h1"], s["h1s"], self.wqkv)
        qkv = s["qkv"].view(self.rows, HQ + 2 * HKV, DH)
        q = P.d3_paged_append(self.cache, qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], self.plan.slots, q=qkv[:, :HQ], rope=self.rope, context=self.plan.context)
        s["att"] = P.d3_paged_attention(self.cache, q, self.plan.table, self.plan.context, rows=self.plan.row, workspace=self.workspace).view(self.rows, HQ * DH)
        s["a8"], s["a8s"] = K.d3_quantize(s["att"])
        s["o"] = K.d3_matmul8(s["a8"], s["a8s"], self.wo, dtype=FP32)
        s["h2"], s["h2s"], s["x2"] = K.d3_add_norm(s["o"], self.norm2, add=self.x)
        s["m"], s["ms"] = K.d3_gated_matmul8(s["h2"], s["h2s"], self.gate, self.up)
        s["d"] = K.d3_matmul8(s["m"], s["ms"], self.down, dtype=FP32)
        s["h3"], s["h3s"], s["x3"] = K.d3_add_norm(s["d"], self.norm3, add=s["x2"])
        s["z"] = K.d3_matmul8(s["h3"], s["h3s"], self.head, dtype=FP32)
        s["out"], s["token"] = K.d3_constrain_logits(s["z"], history=self.history, lengths=self.lengths, repetition=self.repetition, masks=self.masks,
                                                     mask_of=self.mask_of)
        return s

    def check(self, s):
        """Each stage in 64 bits from what the stage before gave."""
        def normed(out, scale, x, gain, add):
            F.check_8_bits(out, scale, *F.norm(x, gain, add, 1e-5)[1:])

        def product(out, a, sc, w):
            F.check_wide(out, *F.product(a, sc, w.q, w.scale))
        normed(s["h1"], s["h1s"], s["x"], self.norm1, None)
        product(s["qkv"], s["h1"], s["h1s"], self.wqkv)
        F.check_8_bits(s["a8"], s["a8s"], s["att"].double(), s["att"].double().abs() * F.U[FP32])
        product(s["o"], s["a8"], s["a8s"], self.wo)
        normed(s["h2"], s["h2s"], s["o"], self.norm2, s["x"])
        g, u = F.product(s["h2"], s["h2s"], self.gate.q, self.gate.scale), F.product(s["h2"], s["h2s"], self.up.q, self.up.scale)
        F.check_8_bits(s["m"], s["ms"], *F.gated(*g, *u))
        product(s["d"], s["m"], s["ms"], self.down)
        normed(s["h3"], s["h3s"], s["d"], self.norm3, s["x2"])
        product(s["z"], s["h3"], s["h3s"], self.head)
        for b in range(self.rows):
            v = s["out"][b]
            top = float(v.max())
            assert int(s["token"][b]) == (-1 if top == float("-inf") else int((v == top).nonzero()[0]))

    def advance(self, token):
        """The chosen tokens are written down and embedded: the next step's input."""
        where = (torch.arange(64, device="cuda") == self.lengths[:, None].long())
        self.history.copy_(torch.where(where, token[:, None], self.history))
        self.lengths += 1
        self.x.copy_(self.embed[token.clamp(min=0).long()])


@pytest.mark.parametrize("rows", [1, 7, 32, 140])
def test_a_block_of_them_eager_and_captured(rows):
    eager, captured = Block(rows), Block(rows)
    start = torch.randn((rows, D), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    eager.x.copy_(start)
    captured.x.copy_(start)
    for step in range(2):                       # (first calls outside of a capture, and the captured one's lengths start at 2)
        a, b = eager.step(), captured.step()
        eager.check(a)
        for name in a:
            assert torch.equal(a[name].view(torch.uint8), b[name].view(torch.uint8)), name
        eager.advance(a["token"])
        captured.advance(b["token"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b = captured.step()
        captured.advance(b["token"])
    for step in range(4):
        a = eager.step()
        eager.check(a)
        held = {k: v.clone() for k, v in a.items()}
        eager.advance(a["token"])
        graph.replay()
        for name in a:
            if name != "x":                     # (advanced inside the graph)
                assert torch.equal(held[name].view(torch.uint8), b[name].view(torch.uint8)), (step, name)


def test_two_streams_at_once():
    g = torch.Generator(device="cuda").manual_seed(1)
    w = K.Weight8(*F.some_weight(4096, 1024, g))
    gate = K.Weight8(*F.some_weight(1000, 1024, g))
    inputs = [F.some_rows(r, 1024, g) for r in (5, 200)]
    want = [(K.d3_matmul8(*i, w, dtype=FP32), *K.d3_gated_matmul8(*i, gate, gate)) for i in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = [[], []]
        for k, st in enumerate(streams):        # one weight, two streams; the results belong to the streams
            got[k] = (K.d3_matmul8(*inputs[k], w, dtype=FP32, stream=st), *K.d3_gated_matmul8(*inputs[k], gate, gate, stream=st))
        torch.cuda.synchronize()
        for k in range(2):
            for a, b in zip(got[k], want[k]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_stream_of_another_device_is_refused():
    class Fake:
        class device:
            index = 1
    w = K.Weight8(*F.some_weight(128, 128, torch.Generator(device="cuda").manual_seed(1)))
    a = F.some_rows(2, 128, torch.Generator(device="cuda").manual_seed(1))
    for call in (lambda: K.d3_matmul8(*a, w, stream=Fake()), lambda: K.d3_quantize(torch.zeros((2, 128), device="cuda"), stream=Fake()),
                 lambda: K.d3_constrain_logits(torch.zeros((2, 128), device="cuda"), stream=Fake())):
        with pytest.raises(K.D3Error):
            call()


def test_what_a_call_writes_counts_as_changed():
    x = torch.randn((4, 256), device="cuda")
    out, total = torch.zeros((4, 256), device="cuda"), torch.zeros((4, 256), device="cuda")
    p = torch.ones((4, 256), device="cuda", requires_grad=True)
    y = (p * out).sum()
    K.d3_add_norm(x, torch.ones(256, device="cuda"), add=x, total=total, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    w = K.d3_quantize_weight(torch.randn((128, 256), device="cuda"))
    version = w.q._version
    K.d3_quantize_weight(torch.randn((128, 256), device="cuda"), out=w)
    assert w.q._version > version
    with torch.inference_mode():
        z = torch.zeros((2, 100), device="cuda")
        K.d3_constrain_logits(z, out=z)
    q, s = K.d3_quantize(x)
    assert not q.requires_grad and not K.d3_matmul8(q, s, w).requires_grad


def test_columns_of_one_buffer():
    """Results go beside what is read, in rows of one buffer."""
    g = torch.Generator(device="cuda").manual_seed(2)
    buf = torch.randn((6, 768), generator=g, device="cuda")
    x, out = buf[:, :256], buf[:, 256:512]
    want, _, _ = K.d3_add_norm(x.clone(), torch.ones(256, device="cuda"), dtype=FP32)
    K.d3_add_norm(x, torch.ones(256, device="cuda"), out=out)
    assert torch.equal(out, want)
    with pytest.raises(K.D3Error):
        K.d3_add_norm(x, torch.ones(256, device="cuda"), out=buf[:, 128:384])
    z = torch.randn((5, 300), generator=g, device="cuda")
    want, token = K.d3_constrain_logits(z[:, :100].clone())
    K.d3_constrain_logits(z[:, :100], out=z[:, 200:])
    assert torch.equal(z[:, 200:], want)
    with pytest.raises(K.D3Error):
        K.d3_constrain_logits(z[:, :100], out=z[:, 50:150])


@pytest.mark.parametrize("rows", [1, 33, 129])
def test_weights_without_a_map_of_their_own(rows):
    """The C ABI encodes a map for the call where the caller has kept none."""
    import ctypes as C
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = K.Weight8(*F.some_weight(260, 272, g))
    a = F.some_rows(rows, 272, g)
    want = K.d3_matmul8(*a, w)
    w.args.map = None
    assert torch.equal(K.d3_matmul8(*a, w), want)
    other = C.create_string_buffer(512)
    bare = K.Weight8Args(C.sizeof(K.Weight8Args), 260, 272, 272, w.q.data_ptr() + 16, w.scale.data_ptr(), (C.addressof(other) + 63) & ~63)
    out = torch.zeros((rows, 260), dtype=BF16, device="cuda")
    args = K.Matmul8Args(C.sizeof(K.Matmul8Args), rows, P.BF16, a[0].data_ptr(), a[1].data_ptr(), out.data_ptr(), None, 272, 3, 260, 0, None)
    assert K.LIB.d3_matmul8(C.byref(bare), C.byref(args), None) == -1       # a map that was not made for this matrix


FIRST = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch, block8_forms as F
from paper_2503_08524_b200 import block8 as K
g = torch.Generator(device="cuda").manual_seed(1)
ws = [K.Weight8(*F.some_weight(n, 1040, g)) for n in (300, 5000)]
a = [F.some_rows(r, 1040, g) for r in (3, 50, 2000)]
x, gain, z = torch.randn((5, 1040), generator=g, device="cuda"), torch.ones(1040, device="cuda"), torch.randn((5, 40000), generator=g, device="cuda")
h = torch.randint(0, 40000, (5, 40000), generator=g, device="cuda").to(torch.int32)
def calls():
    out = [K.d3_matmul8(*i, w) for i in a for w in ws] + [t for i in a for w in ws for t in K.d3_gated_matmul8(*i, w, w)]
    out += list(K.d3_add_norm(x, gain, add=x)) + list(K.d3_quantize(x)) + list(K.d3_constrain_logits(z, history=h)) + list(K.d3_constrain_logits(z, history=h[:, :9]))
    return [t.view(torch.uint8) for t in out]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):          # nothing of this process has run a kernel of these before
    got = calls()
for _ in range(2):
    graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(got, calls()))
print("same")
"""


def test_first_calls_under_capture():
    import os
    import subprocess
    import sys
    tests = os.path.dirname(os.path.abspath(__file__))
    p = subprocess.run([sys.executable, "-c", FIRST.format(root=os.path.dirname(tests), tests=tests)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.strip().endswith("same"), p.stderr[-2000:]
