"""Paged key-value operators of libd3 (include/d3.h): block tables and slot maps from request
lengths, append with rotary positions, attention of one new token per row.

Marshalling only, like `binding`: tensors in, one C call, no host synchronisation; the calls can be
captured into a CUDA graph.  They run on the current stream of the tensors' device unless `stream`
is given.  A refused call raises D3Error (EINVAL) before anything is enqueued; what only the device
can see (a page id out of range, too few free pages) goes to the `status` tensor.

    plan = PagePlan(cached=..., new_tokens=..., table=..., free=..., n_free=..., page_size=..., max_tokens=...)
    plan.d3_page_plan()
    d3_paged_append(cache, k, v, plan.slots, q=q, q_out=q_rot, rope=rope, context=plan.context)
    out = d3_paged_attention(cache, q_rot, plan.table, plan.context, rows=plan.row)
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import EINVAL, LIB, OK, D3Error

BF16, FP16, FP32, E4M3 = 0, 1, 2, 3
MAX_REQUESTS = 4096
_TYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32, torch.float8_e4m3fn: E4M3}

_I32, _I64, _U32, _P = C.c_int32, C.c_int64, C.c_uint32, C.c_void_p


class PagedKVArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + \
        [(n, _I32) for n in ("dtype", "n_pages", "page_size", "n_kv_heads", "head_dim")] + \
        [(n, _I64) for n in ("page_stride", "head_stride", "token_stride")] + \
        [(n, _P) for n in ("k_dev", "v_dev", "k_scale_dev", "v_scale_dev")]


class PagePlanArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + \
        [(n, _I32) for n in ("n_requests", "page_size", "n_pages", "table_width", "max_tokens")] + \
        [("table_stride", _I64)] + \
        [(n, _P) for n in ("cached_dev", "new_tokens_dev", "table_dev", "free_dev", "n_free_dev", "cached_out_dev",
                           "n_free_out_dev", "first_dev", "slots_dev", "row_dev", "context_dev", "status_dev")]


class PagedAppendArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + [(n, _I32) for n in ("dtype", "n_tokens", "n_q_heads", "rope_len")] + \
        [(n, _P) for n in ("k_dev", "v_dev")] + \
        [(n, _I64) for n in ("k_token_stride", "k_head_stride", "v_token_stride", "v_head_stride")] + \
        [(n, _P) for n in ("q_dev", "q_out_dev")] + \
        [(n, _I64) for n in ("q_token_stride", "q_head_stride", "q_out_token_stride", "q_out_head_stride")] + \
        [(n, _P) for n in ("slots_dev", "context_dev", "rope_dev", "status_dev")]


class PagedAttentionArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + \
        [(n, _I32) for n in ("dtype", "n_rows", "n_q_heads", "table_rows", "table_width")] + \
        [("table_stride", _I64), ("scale", C.c_float), ("q_dev", _P), ("q_row_stride", _I64), ("q_head_stride", _I64),
         ("out_dev", _P), ("out_row_stride", _I64), ("out_head_stride", _I64), ("lse_dev", _P), ("table_dev", _P),
         ("context_dev", _P), ("rows_dev", _P), ("workspace_dev", _P), ("workspace_bytes", C.c_size_t),
         ("status_dev", _P)]


def _refuse(what: str):
    raise D3Error(EINVAL, what)


def _strides(t: torch.Tensor):
    """Strides of all dimensions but the last; those of a dimension of one entry (which torch leaves
    arbitrary) as if the tensor were contiguous there."""
    st, inner = list(t.stride()), 1
    for d in range(t.dim() - 1, -1, -1):
        if t.shape[d] <= 1:
            st[d] = inner
        inner = max(inner, st[d] * t.shape[d])
    return st[:-1]


def _call(fn, what: str, device: torch.device, stream, *args) -> None:
    """One C call on `stream` (default: the device's current stream), with the device current."""
    if device.type != "cuda":
        _refuse(what + ": tensors must be on a CUDA device")
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        _refuse(what + ": stream of another device")
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, stream.cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream.cuda_stream)
    if rc != OK:
        raise D3Error(rc, what)


def _vector(t: torch.Tensor, dtype, n: Optional[int], device, what: str) -> int:
    """Data pointer of a contiguous 1-D tensor of `n` entries (None: any number)."""
    if t.dtype != dtype or t.dim() != 1 or (n is not None and t.shape[0] != n) or t.device != device or not t.is_contiguous():
        _refuse(f"{what}: expected a contiguous {dtype} vector" + ("" if n is None else f" of {n}") + f" on {device}")
    return t.data_ptr()


def _status(t: Optional[torch.Tensor], device, what: str):
    return None if t is None else _vector(t, torch.int32, 1, device, what + " status")


class PagedKV:
    """A pool of pages.  k, v: [n_pages][n_kv_heads][page_size][head_dim] with equal strides, head_dim
    contiguous (a pool kept token by token is passed as `t.permute(0, 2, 1, 3)`); bf16, fp16 or
    float8_e4m3fn.  k_scale, v_scale (8-bit pools): fp32 [n_kv_heads]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        if k.dim() != 4 or k.shape != v.shape or _strides(k) != _strides(v) or k.dtype != v.dtype or k.device != v.device:
            _refuse("PagedKV: k and v must be 4-D tensors of one shape, type, device and stride")
        if k.dtype not in _TYPES or k.dtype == torch.float32 or k.stride(3) != 1:
            _refuse("PagedKV: bf16, fp16 or float8_e4m3fn with contiguous head_dim")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.dtype = k.device, k.dtype
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        sc = [None if s is None else _vector(s, torch.float32, self.n_kv_heads, k.device, "PagedKV scale")
              for s in (k_scale, v_scale)]
        if k.dtype != torch.float8_e4m3fn and (k_scale is not None or v_scale is not None):
            _refuse("PagedKV: scales belong to an 8-bit pool")
        st = _strides(k)
        self.args = PagedKVArgs(C.sizeof(PagedKVArgs), _TYPES[k.dtype], self.n_pages, self.page_size, self.n_kv_heads,
                                self.head_dim, st[0], st[1], st[2], k.data_ptr(), v.data_ptr(), sc[0], sc[1])
        self._ref = C.byref(self.args)
        n = C.c_size_t()   # the sizes this library serves
        if LIB.d3_paged_attention_workspace(self._ref, self.n_kv_heads, C.byref(n)) != OK:
            _refuse("PagedKV: page_size a power of two in 16..1024, head_dim 32, 64 or 128")


def model_view(model, layer: int):
    """See D3Model.d3_paged_view."""
    kv, table, rows, width = PagedKVArgs(), _P(), _I32(), _I32()
    rc = LIB.d3_paged_view(model.h, layer, C.byref(kv), C.byref(table), C.byref(rows), C.byref(width))
    if rc != OK:
        raise D3Error(rc, "d3_paged_view")
    shape = (kv.n_pages, kv.n_kv_heads, kv.page_size, kv.head_dim)
    n = kv.n_pages * kv.page_stride
    cells = model.kv.view(torch.bfloat16)
    k0 = (kv.k_dev - model.kv.data_ptr()) // 2
    v0 = (kv.v_dev - model.kv.data_ptr()) // 2
    t0 = table.value - model.scratch.data_ptr()
    entries = model.scratch[t0:t0 + 4 * rows.value * width.value].view(torch.int32).view(rows.value, width.value)
    return PagedKV(cells[k0:k0 + n].view(shape), cells[v0:v0 + n].view(shape)), entries


class PagePlan:
    """d3_page_plan over fixed tensors (see include/d3.h), as a serving loop or a captured graph holds them.

    cached, new_tokens [n_requests], free [n_pages], n_free [1]: int32; table: int32 [n_requests][width].
    cached_out, n_free_out default to cached and n_free themselves (lengths advance in place).  Outputs:
    .slots int64, .row, .context int32 [max_tokens]; .first int32 [n_requests + 1]; .status int32 [1]."""

    def __init__(self, *, cached: torch.Tensor, new_tokens: torch.Tensor, table: torch.Tensor, free: torch.Tensor,
                 n_free: torch.Tensor, page_size: int, max_tokens: int, cached_out: Optional[torch.Tensor] = None,
                 n_free_out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
        dev, what = cached.device, "PagePlan"
        R = cached.shape[0] if cached.dim() == 1 else -1
        if not (1 <= R <= MAX_REQUESTS) or max_tokens < 1 or max_tokens > 0x7fffffff:
            _refuse(f"{what}: 1..{MAX_REQUESTS} requests, max_tokens >= 1")
        if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != R or table.device != dev or \
                table.stride(1) != 1 or table.shape[1] < 1 or (R > 1 and table.stride(0) < table.shape[1]):
            _refuse(f"{what}: table must be int32 [n_requests][width] on {dev}")
        self.cached, self.new_tokens, self.table, self.free, self.n_free = cached, new_tokens, table, free, n_free
        self.cached_out = cached if cached_out is None else cached_out
        self.n_free_out = n_free if n_free_out is None else n_free_out
        self.device = dev
        self.slots = torch.empty(max_tokens, dtype=torch.int64, device=dev)
        self.row = torch.empty(max_tokens, dtype=torch.int32, device=dev)
        self.context = torch.empty(max_tokens, dtype=torch.int32, device=dev)
        self.first = torch.empty(R + 1, dtype=torch.int32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev) if status is None else status
        i32 = torch.int32
        self.args = PagePlanArgs(
            C.sizeof(PagePlanArgs), R, page_size, free.shape[0] if free.dim() == 1 else 0, table.shape[1], max_tokens,
            table.stride(0) if R > 1 else table.shape[1], _vector(cached, i32, R, dev, what + " cached"),
            _vector(new_tokens, i32, R, dev, what + " new_tokens"), table.data_ptr(), _vector(free, i32, None, dev, what + " free"),
            _vector(n_free, i32, 1, dev, what + " n_free"), _vector(self.cached_out, i32, R, dev, what + " cached_out"),
            _vector(self.n_free_out, i32, 1, dev, what + " n_free_out"), self.first.data_ptr(), self.slots.data_ptr(),
            self.row.data_ptr(), self.context.data_ptr(), _status(self.status, dev, what))
        self._ref = C.byref(self.args)

    def d3_page_plan(self, stream=None) -> "PagePlan":
        _call(LIB.d3_page_plan, "d3_page_plan", self.device, stream, self._ref)
        return self


def _heads(t: torch.Tensor, n: int, heads: int, dh: int, dtype, device, what: str):
    """[n][heads][dh] with dh contiguous."""
    if t.shape != (n, heads, dh) or t.dtype != dtype or t.device != device or t.stride(2) != 1:
        _refuse(f"{what}: expected {dtype} [{n}][{heads}][{dh}] on {device}, last dimension contiguous")


def d3_rope_table(n_positions: int, head_dim: int, base: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    """fp32 [n_positions][head_dim / 2][2]: (cos, sin) of position * base^(-2j / head_dim), angles in fp64."""
    dev = torch.device(device)
    if dev.index is None and dev.type == "cuda":
        dev = torch.device("cuda", torch.cuda.current_device())
    if n_positions < 1 or head_dim not in (32, 64, 128):
        _refuse("d3_rope_table: n_positions >= 1, head_dim 32, 64 or 128")
    t = torch.empty((n_positions, head_dim // 2, 2), dtype=torch.float32, device=dev)
    _call(LIB.d3_rope_table, "d3_rope_table", dev, stream, n_positions, head_dim, float(base), t.data_ptr())
    return t


def d3_paged_append(cache: PagedKV, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
                    q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                    rope: Optional[torch.Tensor] = None, context: Optional[torch.Tensor] = None,
                    status: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """k, v [n][n_kv_heads][head_dim] to the slots (int64 [n], negative = padding); with `rope`, k is
    rotated by position context - 1 and q [n][n_q_heads][head_dim] goes rotated to q_out (default: a
    new tensor whose padding rows are undefined; q itself is allowed).  Returns q_out."""
    what, dev = "d3_paged_append", cache.device
    n, hkv, dh = slots.shape[0] if slots.dim() == 1 else -1, cache.n_kv_heads, cache.head_dim
    if k.dtype not in _TYPES:
        _refuse(f"{what}: unsupported type {k.dtype}")
    _heads(k, n, hkv, dh, k.dtype, dev, what + " k")
    _heads(v, n, hkv, dh, k.dtype, dev, what + " v")
    a = PagedAppendArgs()
    a.struct_size, a.dtype, a.n_tokens = C.sizeof(PagedAppendArgs), _TYPES[k.dtype], n
    a.slots_dev = _vector(slots, torch.int64, n, dev, what + " slots")
    a.k_dev, a.v_dev = k.data_ptr(), v.data_ptr()
    a.k_token_stride, a.k_head_stride = _strides(k)
    a.v_token_stride, a.v_head_stride = _strides(v)
    if rope is not None:
        if rope.dtype != torch.float32 or rope.dim() != 3 or rope.shape[1:] != (dh // 2, 2) or rope.device != dev or \
                not rope.is_contiguous():
            _refuse(f"{what}: rope must be contiguous fp32 [positions][{dh // 2}][2] on {dev}")
        if context is None:
            _refuse(f"{what}: rope needs context")
        a.rope_dev, a.rope_len = rope.data_ptr(), rope.shape[0]
        a.context_dev = _vector(context, torch.int32, n, dev, what + " context")
    if q is not None:
        if rope is None:
            _refuse(f"{what}: q is only rotated, and there is no rope")
        hq = q.shape[1] if q.dim() == 3 else -1
        _heads(q, n, hq, dh, k.dtype, dev, what + " q")
        if q_out is None:
            q_out = torch.empty((n, hq, dh), dtype=k.dtype, device=dev)
        _heads(q_out, n, hq, dh, k.dtype, dev, what + " q_out")
        a.n_q_heads, a.q_dev, a.q_out_dev = hq, q.data_ptr(), q_out.data_ptr()
        a.q_token_stride, a.q_head_stride = _strides(q)
        a.q_out_token_stride, a.q_out_head_stride = _strides(q_out)
    elif q_out is not None:
        _refuse(f"{what}: q_out without q")
    if status is not None:
        a.status_dev = _status(status, dev, what)
    if n > 0:
        _call(LIB.d3_paged_append, what, dev, stream, cache._ref, C.byref(a))
    return q_out


def attention_workspace(cache: PagedKV, n_q_heads: int) -> torch.Tensor:
    """Workspace of d3_paged_attention calls over `cache` that do not overlap."""
    n = C.c_size_t()
    rc = LIB.d3_paged_attention_workspace(cache._ref, n_q_heads, C.byref(n))
    if rc != OK:
        raise D3Error(rc, "d3_paged_attention_workspace")
    return torch.empty(n.value, dtype=torch.uint8, device=cache.device)


def d3_paged_attention(cache: PagedKV, q: torch.Tensor, table: torch.Tensor, context: torch.Tensor, *,
                       rows: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                       out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, with_lse: bool = False,
                       workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None):
    """q [n][n_q_heads][head_dim] over the first context[b] positions of the pages that
    table[rows[b] or b] names (see include/d3.h).  scale: default head_dim^-0.5.  Returns out, or
    (out, lse) with `with_lse` or an `lse` tensor (fp32 [n][n_q_heads]).  Without `workspace` one is allocated for the
    call."""
    what, dev = "d3_paged_attention", cache.device
    if q.dim() != 3 or q.dtype not in _TYPES:
        _refuse(f"{what}: q must be [n][n_q_heads][head_dim]")
    n, hq, dh = q.shape
    _heads(q, n, hq, cache.head_dim, q.dtype, dev, what + " q")
    if table.dtype != torch.int32 or table.dim() != 2 or table.device != dev or table.shape[0] < 1 or table.shape[1] < 1 or \
            table.stride(1) != 1:
        _refuse(f"{what}: table must be int32 [rows][width] on {dev}")
    if out is None:
        out = torch.empty((n, hq, dh), dtype=q.dtype, device=dev)
    else:
        _heads(out, n, hq, dh, q.dtype, dev, what + " out")
    if lse is None:
        if with_lse:
            lse = torch.empty((n, hq), dtype=torch.float32, device=dev)
    elif lse.shape != (n, hq) or lse.dtype != torch.float32 or lse.device != dev or not lse.is_contiguous():
        _refuse(f"{what}: lse must be contiguous fp32 [{n}][{hq}] on {dev}")
    if workspace is None:
        workspace = attention_workspace(cache, hq)
    elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
        _refuse(f"{what}: workspace must be contiguous uint8 on {dev}")
    qs, os = _strides(q), _strides(out)
    a = PagedAttentionArgs(
        C.sizeof(PagedAttentionArgs), _TYPES[q.dtype], n, hq, table.shape[0], table.shape[1],
        table.stride(0) if table.shape[0] > 1 else table.shape[1], dh ** -0.5 if scale is None else scale, q.data_ptr(), qs[0], qs[1],
        out.data_ptr(), os[0], os[1], None if lse is None else lse.data_ptr(), table.data_ptr(),
        _vector(context, torch.int32, n, dev, what + " context"),
        None if rows is None else _vector(rows, torch.int32, n, dev, what + " rows"),
        workspace.data_ptr(), workspace.numel(), _status(status, dev, what))
    if n > 0:
        _call(LIB.d3_paged_attention, what, dev, stream, cache._ref, C.byref(a))
    return out if lse is None else (out, lse)
