"""8-bit block operators of libd3 (include/d3.h): norm with the residual's sum and a result in 8 bits, products of 8-bit
rows and weights, the gated pair of them, and the constraints that stand between logits and a token.

With the paged operators (`paged`) they make up a decoder block for callers that run one themselves:

    wqkv, wo, w_gate, w_up, w_down = (d3_quantize_weight(w) for w in ...)                   # once
    h, hs, _ = d3_add_norm(x, attn_norm)                                                      # x: the residual stream
    qkv = d3_matmul8(h, hs, wqkv)
    ...                                                                                       # paged append and attention
    o = d3_matmul8(*d3_quantize(att), wo)
    h, hs, x = d3_add_norm(o, mlp_norm, add=x, total=x)
    y = d3_matmul8(*d3_gated_matmul8(h, hs, w_gate, w_up), w_down)
    ...
    logits, token = d3_constrain_logits(logits, history=tokens, lengths=n, repetition=r, masks=grammar, mask_of=state)

Marshalling only, like `paged` (the checks of a call are in csrc/block_call.cpp): tensors in, one C call, no host
synchronisation; the calls can be captured into a CUDA graph.  They run on the current stream of the tensors' device unless
`stream` is given.  Results carry no gradient; what a call writes into counts as changed in place.  A refused call raises
D3Error (EINVAL) before anything is enqueued; what only the device can see (a token id out of range, a wait that ran out)
goes to the `status` tensor.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import build as _build
from .binding import EINVAL, LIB, OK, D3Error
from .paged import _TYPES, _on_stream, _refuse

_block_call = _build.load_call("block_call")
_block_call.bind(*[C.cast(f, C.c_void_p).value for f in (LIB.d3_add_norm, LIB.d3_matmul8, LIB.d3_gated_matmul8, LIB.d3_constrain_logits)],
                 D3Error)

BLOCK, MAP_BYTES = 128, 256

_I32, _I64, _U32, _P = C.c_int32, C.c_int64, C.c_uint32, C.c_void_p


class Weight8Args(C.Structure):
    _fields_ = [("struct_size", _U32), ("n", _I32), ("k", _I32), ("row_stride", _I64), ("q_dev", _P), ("scale_dev", _P), ("map", _P)]


class AddNormArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + \
        [(n, _I32) for n in ("n_rows", "dim", "x_dtype", "add_dtype", "gain_dtype", "out_dtype")] + [("eps", C.c_float)] + \
        [(n, _P) for n in ("x_dev", "add_dev", "total_dev", "gain_dev", "out_dev", "scale_dev")] + \
        [(n, _I64) for n in ("x_stride", "add_stride", "total_stride", "out_stride", "scale_stride")]


class Matmul8Args(C.Structure):
    _fields_ = [("struct_size", _U32), ("n_rows", _I32), ("out_dtype", _I32)] + \
        [(n, _P) for n in ("a_dev", "a_scale_dev", "out_dev", "scale_dev")] + \
        [(n, _I64) for n in ("a_stride", "a_scale_stride", "out_stride", "scale_stride")] + [("status_dev", _P)]


class ConstrainLogitsArgs(C.Structure):
    _fields_ = [("struct_size", _U32)] + [(n, _I32) for n in ("dtype", "n_rows", "vocab", "n_history", "n_bias", "n_masks")] + \
        [(n, _P) for n in ("logits_dev", "out_dev")] + \
        [(n, _I64) for n in ("logits_stride", "out_stride", "history_stride", "bias_stride", "mask_stride")] + \
        [(n, _P) for n in ("history_dev", "lengths_dev", "prompt_dev", "repetition_dev", "frequency_dev", "presence_dev",
                           "bias_ids_dev", "bias_dev", "masks_dev", "mask_of_dev", "token_dev", "status_dev")]


def _blocks(n: int) -> int:
    return -(-n // BLOCK)


class Weight8:
    """A weight matrix in 8 bits: q float8_e4m3fn [n][k] (k a multiple of 16, rows contiguous and 16-byte aligned), scale
    fp32 [ceil(n / 128)][ceil(k / 128)], contiguous: the value of q[i][j] is q[i][j] * scale[i // 128][j // 128]."""

    def __init__(self, q: torch.Tensor, scale: torch.Tensor):
        if q.dim() != 2 or q.dtype != torch.float8_e4m3fn or q.shape[0] < 1 or q.shape[1] < 16 or q.shape[1] % 16 or q.stride(1) != 1:
            _refuse("Weight8: q must be float8_e4m3fn [n][k] with contiguous rows, k a multiple of 16")
        n, k = q.shape
        stride = q.stride(0) if n > 1 else k
        if scale.dtype != torch.float32 or tuple(scale.shape) != (_blocks(n), _blocks(k)) or not scale.is_contiguous() or scale.device != q.device:
            _refuse(f"Weight8: scale must be contiguous fp32 [{_blocks(n)}][{_blocks(k)}] on {q.device}")
        if stride % 16 or stride < k or q.data_ptr() % 16:
            _refuse("Weight8: rows of q must start on 16 bytes and not overlap")
        self.q, self.scale, self.n, self.k = q, scale, n, k
        self.device, self.index = q.device, q.get_device()
        self.args = Weight8Args(C.sizeof(Weight8Args), n, k, stride, q.data_ptr(), scale.data_ptr(), None)
        self._ref, self._at = C.byref(self.args), C.addressof(self.args)
        if self.index >= 0:   # the matrix' tensor map, encoded once
            self._map = C.create_string_buffer(MAP_BYTES + 64)
            at = (C.addressof(self._map) + 63) & ~63
            rc = LIB.d3_weight8_map(self._ref, at)
            if rc != OK:
                raise D3Error(rc, "Weight8")
            self.args.map = at


def d3_quantize_weight(w: torch.Tensor, *, out: Optional[Weight8] = None, stream=None) -> Weight8:
    """w [n][k] (bf16, fp16 or fp32, rows contiguous, k a multiple of 16) in 8 bits, a scale for each block of 128 x 128.
    `out`: a Weight8 of that shape to write into."""
    what = "d3_quantize_weight"
    if w.dim() != 2 or w.dtype not in (torch.bfloat16, torch.float16, torch.float32) or w.shape[0] < 1 or w.shape[1] < 16 or w.shape[1] % 16 or \
            w.stride(1) != 1 or not w.is_cuda:
        _refuse(f"{what}: w must be bf16, fp16 or fp32 [n][k] with contiguous rows on a CUDA device, k a multiple of 16")
    if stream is not None:
        return _on_stream(lambda: d3_quantize_weight(w, out=out), w.get_device(), stream, what)
    n, k = w.shape
    if out is None:
        out = Weight8(torch.empty((n, k), dtype=torch.float8_e4m3fn, device=w.device),
                      torch.empty((_blocks(n), _blocks(k)), dtype=torch.float32, device=w.device))
    elif (out.n, out.k, out.device) != (n, k, w.device):
        _refuse(f"{what}: out must be [{n}][{k}] on {w.device}")
    with torch.cuda.device(w.device):
        rc = LIB.d3_quantize_weight(w.data_ptr(), _TYPES[w.dtype], w.stride(0) if n > 1 else k, out._ref,
                                    torch.cuda.current_stream(w.device).cuda_stream)
    if rc != OK:
        raise D3Error(rc, what)
    for t in (out.q, out.scale):
        if not t.is_inference():
            torch.autograd.graph.increment_version(t)
    return out


def d3_add_norm(x: torch.Tensor, gain: Optional[torch.Tensor], *, add: Optional[torch.Tensor] = None, total: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
                eps: float = 1e-5, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """RMSNorm of x + add (see include/d3.h); x [rows][dim], gain [dim] (None: no norm), add of x's type or fp32.  Returns
    (out, scale, total): out in `dtype` (float8_e4m3fn unless it or `out` says otherwise) with its scale fp32
    [rows][ceil(dim / 128)] (None for wider types), and the sum in add's type (None without add; total=add: in place)."""
    if stream is not None:
        return _on_stream(lambda: d3_add_norm(x, gain, add=add, total=total, out=out, scale=scale, dtype=dtype, eps=eps), x.get_device(),
                          stream, "d3_add_norm")
    return _block_call.norm("d3_add_norm", x, gain, add, total, out, scale, dtype, eps)


def d3_quantize(x: torch.Tensor, *, out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows of x in 8 bits with a scale for each 128 numbers: (float8_e4m3fn [rows][dim], fp32 [rows][ceil(dim / 128)])."""
    if stream is not None:
        return _on_stream(lambda: d3_quantize(x, out=out, scale=scale), x.get_device(), stream, "d3_quantize")
    return _block_call.norm("d3_quantize", x, None, None, None, out, scale, torch.float8_e4m3fn, 0.0)[:2]


def d3_matmul8(a: torch.Tensor, a_scale: torch.Tensor, weight: Weight8, *, out: Optional[torch.Tensor] = None,
               dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """a [rows][k] float8_e4m3fn with a_scale times weight [n][k] transposed: [rows][n] in `dtype` (default bf16, or out's)."""
    if stream is not None:
        return _on_stream(lambda: d3_matmul8(a, a_scale, weight, out=out, dtype=dtype, status=status), weight.index, stream, "d3_matmul8")
    return _block_call.product(weight._at, 0, weight.index, a, a_scale, out, None, dtype, status)


def d3_gated_matmul8(a: torch.Tensor, a_scale: torch.Tensor, gate: Weight8, up: Weight8, *, out: Optional[torch.Tensor] = None,
                     scale: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """silu(a gate^T) * (a up^T): (out [rows][n] in `dtype` (default float8_e4m3fn, or out's), its scale fp32
    [rows][ceil(n / 128)], None for wider types)."""
    if gate.index != up.index:
        _refuse("d3_gated_matmul8: both weights must be on one device")
    if stream is not None:
        return _on_stream(lambda: d3_gated_matmul8(a, a_scale, gate, up, out=out, scale=scale, dtype=dtype, status=status), gate.index, stream,
                          "d3_gated_matmul8")
    return _block_call.product(gate._at, up._at, gate.index, a, a_scale, out, scale, dtype, status)


def d3_matmul8_plan(rows: int, n: int, k: int, gated: bool = False) -> Tuple[int, int]:
    """How a product of these sizes is done: (rows of a tile: 16 to 128, or 256 in the kernel for many rows; CTAs that share its k)."""
    plan = (_I32 * 2)()
    rc = LIB.d3_matmul8_plan(rows, n, k, int(bool(gated)), plan)
    if rc != OK:
        raise D3Error(rc, "d3_matmul8_plan")
    return plan[0], plan[1]


def d3_matmul8_set_wait_ns(ns: int) -> None:
    """Limit of every wait inside the products of this process from now on (default 2e9)."""
    rc = LIB.d3_matmul8_set_wait_ns(int(ns)) if int(ns) >= 0 else EINVAL
    if rc != OK:
        raise D3Error(rc, "d3_matmul8_set_wait_ns")


def d3_matmul8_stall_next(on: int) -> None:
    """Drill: the waits for copies of the next product cannot be satisfied (1; 0: none)."""
    rc = LIB.d3_matmul8_stall_next(int(on))
    if rc != OK:
        raise D3Error(rc, "d3_matmul8_stall_next")


def d3_constrain_logits(logits: torch.Tensor, *, history: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                        prompt: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                        frequency: Optional[torch.Tensor] = None, presence: Optional[torch.Tensor] = None,
                        bias_ids: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                        masks: Optional[torch.Tensor] = None, mask_of: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(logits [rows][vocab] with penalties, biases and masks applied, best token int32 [rows]); see include/d3.h.  history
    int32 [rows][n] (negative: padding), lengths, prompt int32 [rows]; repetition, frequency, presence fp32 [rows]; bias_ids
    int32 and bias fp32 [rows][m]; masks int32 [states][ceil(vocab / 32)] (bit set: allowed), mask_of int32 [rows] (-1: none).
    out=logits works in place."""
    if stream is not None:
        return _on_stream(lambda: d3_constrain_logits(logits, history=history, lengths=lengths, prompt=prompt, repetition=repetition,
                                                      frequency=frequency, presence=presence, bias_ids=bias_ids, bias=bias, masks=masks,
                                                      mask_of=mask_of, out=out, token=token, status=status),
                          logits.get_device(), stream, "d3_constrain_logits")
    return _block_call.logits(logits, history, lengths, prompt, repetition, frequency, presence, bias_ids, bias, masks, mask_of, out, token,
                              status)
