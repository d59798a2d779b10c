"""Paged key-value operators of libd3 (include/d3.h): block tables and slot maps from request
lengths, append with rotary positions, attention of one new token per row.

Marshalling only, like `binding`: tensors in, one C call, no host synchronisation; the calls can be
captured into a CUDA graph.  The checks of each call are in csrc/paged_call.cpp (a small decode step is
bound by the host side of its calls).  They run on the current stream of the tensors' device unless `stream`
is given.  Results carry no gradient; what a call writes into counts as changed in place.  A refused call raises D3Error (EINVAL) before anything is enqueued; what only the device
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

from . import build as _build
from .binding import EINVAL, LIB, OK, D3Error

_paged_call = _build.load_call()
_paged_call.bind(*[C.cast(f, C.c_void_p).value for f in (LIB.d3_page_plan, LIB.d3_paged_append, LIB.d3_paged_attention,
                                                         LIB.d3_paged_attention_workspace)], D3Error)

BF16, FP16, FP32, E4M3 = 0, 1, 2, 3
STALL_COPIES, STALL_SUMS = 1, 2
MAX_REQUESTS, MAPS_BYTES = 4096, 640
_TYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32, torch.float8_e4m3fn: E4M3}

_I32, _I64, _U32, _P = C.c_int32, C.c_int64, C.c_uint32, C.c_void_p


class PagedKVArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + \
        [(n, _I32) for n in ("dtype", "n_pages", "page_size", "n_kv_heads", "head_dim")] + \
        [(n, _I64) for n in ("page_stride", "head_stride", "token_stride")] + \
        [(n, _P) for n in ("k_dev", "v_dev", "k_scale_dev", "v_scale_dev", "maps")]


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


def _on_stream(call, index: int, stream, what: str):
    """`call` with `stream` current, so that what it allocates belongs to that stream."""
    if index < 0 or stream.device.index != index:
        _refuse(f"{what}: stream and tensors must be on one CUDA device")
    with torch.cuda.stream(stream):
        return call()


def _vector(t: torch.Tensor, dtype, n: int, index: int, what: str, name: str) -> int:
    """Data pointer of a contiguous 1-D tensor of `n` entries (-1: any number)."""
    if t.dtype is not dtype or t.get_device() != index or t.dim() != 1 or (t.shape[0] != n and n != -1) or not t.is_contiguous():
        _refuse(f"{what}: {name} must be a contiguous {dtype} vector" + ("" if n < 0 else f" of {n}") + f" on device {index}")
    return t.data_ptr()


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
        self.device, self.dtype, self.index = k.device, k.dtype, k.get_device()
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        sc = [None if s is None else _vector(s, torch.float32, self.n_kv_heads, self.index, "PagedKV", "scale")
              for s in (k_scale, v_scale)]
        if k.dtype != torch.float8_e4m3fn and (k_scale is not None or v_scale is not None):
            _refuse("PagedKV: scales belong to an 8-bit pool")
        st = _strides(k)
        self.args = PagedKVArgs(C.sizeof(PagedKVArgs), _TYPES[k.dtype], self.n_pages, self.page_size, self.n_kv_heads,
                                self.head_dim, st[0], st[1], st[2], k.data_ptr(), v.data_ptr(), sc[0], sc[1], None)
        self._ref, self._at = C.byref(self.args), C.addressof(self.args)
        n = C.c_size_t()   # the sizes this library serves
        if LIB.d3_paged_attention_workspace(self._ref, self.n_kv_heads, C.byref(n)) != OK:
            _refuse("PagedKV: page_size a power of two in 16..1024, head_dim 32, 64 or 128")
        if self.index >= 0:   # the pool's tensor maps, encoded once
            self._maps = C.create_string_buffer(MAPS_BYTES + 64)
            maps = (C.addressof(self._maps) + 63) & ~63
            rc = LIB.d3_paged_maps(self._ref, maps)
            if rc != OK:
                raise D3Error(rc, "PagedKV")
            self.args.maps = maps


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
        dev, index, what, i32 = cached.device, cached.get_device(), "PagePlan", torch.int32
        R = cached.shape[0] if cached.dim() == 1 else -1
        if not (1 <= R <= MAX_REQUESTS) or not (1 <= max_tokens <= 0x7fffffff):
            _refuse(f"{what}: 1..{MAX_REQUESTS} requests, max_tokens >= 1")
        if table.dtype != i32 or table.dim() != 2 or table.shape[0] != R or table.device != dev or table.shape[1] < 1 or \
                (table.shape[1] > 1 and table.stride(1) != 1):
            _refuse(f"{what}: table must be int32 [n_requests][width] on {dev}")
        self.cached, self.new_tokens, self.table, self.free, self.n_free = cached, new_tokens, table, free, n_free
        self.cached_out = cached if cached_out is None else cached_out
        self.n_free_out = n_free if n_free_out is None else n_free_out
        self.index = index
        self.slots = torch.empty(max_tokens, dtype=torch.int64, device=dev)
        self.row = torch.empty(max_tokens, dtype=i32, device=dev)
        self.context = torch.empty(max_tokens, dtype=i32, device=dev)
        self.first = torch.empty(R + 1, dtype=i32, device=dev)
        self.status = torch.zeros(1, dtype=i32, device=dev) if status is None else status
        self.args = PagePlanArgs(
            C.sizeof(PagePlanArgs), R, page_size, free.shape[0] if free.dim() == 1 else 0, table.shape[1], max_tokens,
            table.stride(0) if R > 1 else table.shape[1], _vector(cached, i32, R, index, what, "cached"),
            _vector(new_tokens, i32, R, index, what, "new_tokens"), table.data_ptr(), _vector(free, i32, -1, index, what, "free"),
            _vector(n_free, i32, 1, index, what, "n_free"), _vector(self.cached_out, i32, R, index, what, "cached_out"),
            _vector(self.n_free_out, i32, 1, index, what, "n_free_out"), self.first.data_ptr(), self.slots.data_ptr(),
            self.row.data_ptr(), self.context.data_ptr(), _vector(self.status, i32, 1, index, what, "status"))
        self._at = C.addressof(self.args)
        self._written = (table, free, self.cached_out, self.n_free_out, self.slots, self.row, self.context, self.first)

    def d3_page_plan(self, stream=None) -> "PagePlan":
        if stream is not None:
            return _on_stream(self.d3_page_plan, self.index, stream, "d3_page_plan")
        _paged_call.plan(self._at, self.index, self._written)
        return self


def d3_rope_table(n_positions: int, head_dim: int, base: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    """fp32 [n_positions][head_dim / 2][2]: (cos, sin) of position * base^(-2j / head_dim), angles in fp64."""
    dev = torch.device(device)
    if dev.index is None and dev.type == "cuda":
        dev = torch.device("cuda", torch.cuda.current_device())
    if n_positions < 1 or head_dim not in (32, 64, 128):
        _refuse("d3_rope_table: n_positions >= 1, head_dim 32, 64 or 128")
    if stream is not None:
        return _on_stream(lambda: d3_rope_table(n_positions, head_dim, base, dev), -1 if dev.type != "cuda" else dev.index, stream,
                          "d3_rope_table")
    t = torch.empty((n_positions, head_dim // 2, 2), dtype=torch.float32, device=dev)
    if dev.type != "cuda":
        _refuse("d3_rope_table: a CUDA device")
    with torch.cuda.device(dev):
        rc = LIB.d3_rope_table(n_positions, head_dim, float(base), t.data_ptr(), torch.cuda.current_stream(dev).cuda_stream)
    if rc != OK:
        raise D3Error(rc, "d3_rope_table")
    return t


def d3_paged_append(cache: PagedKV, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
                    q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                    rope: Optional[torch.Tensor] = None, context: Optional[torch.Tensor] = None,
                    status: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """k, v [n][n_kv_heads][head_dim] to the slots (int64 [n], negative = padding); with `rope`, k is
    rotated by position context - 1 and q [n][n_q_heads][head_dim] goes rotated to q_out (default: a
    new tensor whose padding rows are undefined; q itself is allowed).  Returns q_out."""
    if stream is not None:
        return _on_stream(lambda: d3_paged_append(cache, k, v, slots, q=q, q_out=q_out, rope=rope, context=context, status=status),
                          cache.index, stream, "d3_paged_append")
    return _paged_call.append(cache._at, cache.index, k, v, slots, q, q_out, rope, context, status, cache.k, cache.v)


def attention_workspace(cache: PagedKV, n_q_heads: int) -> torch.Tensor:
    """Workspace of d3_paged_attention calls over `cache` that do not overlap."""
    n = C.c_size_t()
    rc = LIB.d3_paged_attention_workspace(cache._ref, n_q_heads, C.byref(n))
    if rc != OK:
        raise D3Error(rc, "d3_paged_attention_workspace")
    return torch.empty(n.value, dtype=torch.uint8, device=cache.device)


def d3_paged_set_wait_ns(ns: int) -> None:
    """Limit of every wait inside the d3_paged_attention calls of this process from now on (default 2e9)."""
    rc = LIB.d3_paged_set_wait_ns(int(ns)) if int(ns) >= 0 else EINVAL
    if rc != OK:
        raise D3Error(rc, "d3_paged_set_wait_ns")


def d3_paged_stall_next(what: int) -> None:
    """Drill: a wait of the next d3_paged_attention call cannot be satisfied (STALL_COPIES, STALL_SUMS; 0: none)."""
    rc = LIB.d3_paged_stall_next(int(what))
    if rc != OK:
        raise D3Error(rc, "d3_paged_stall_next")


def d3_paged_attention(cache: PagedKV, q: torch.Tensor, table: torch.Tensor, context: torch.Tensor, *,
                       rows: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                       out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, with_lse: bool = False,
                       workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None):
    """q [n][n_q_heads][head_dim] over the first context[b] positions of the pages that
    table[rows[b] or b] names (see include/d3.h).  scale: default head_dim^-0.5.  Returns out (default: a new
    tensor whose padding rows are undefined), or (out, lse) with `with_lse` or an `lse` tensor (fp32 [n][n_q_heads]).  Without `workspace` one is allocated for the
    call."""
    if stream is not None:
        return _on_stream(lambda: d3_paged_attention(cache, q, table, context, rows=rows, scale=scale, out=out, lse=lse,
                                                     with_lse=with_lse, workspace=workspace, status=status),
                          cache.index, stream, "d3_paged_attention")
    return _paged_call.attention(cache._at, cache.index, q, table, context, rows, scale, out, lse, with_lse, workspace, status)
