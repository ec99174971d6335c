"""What stands around a worker's attention, on torch tensors: norms with gate
and residual, products in 8-bit integers, and linear attention over a pool of
states (``kvr_block_norm``, ``kvr_integer_product`` and
``kvr_linear_attention`` of include/kvr.h, which says what they compute).

As in ``serve``: the functions check what the C side cannot see (types, shapes,
devices), marshal the arguments and launch on torch's current stream of the
tensors' device; they neither synchronise nor copy to the host; errors raise
``KvrError``; there are no gradients, and a call whose result would need one, or
would have a tangent, is refused.
"""
from __future__ import annotations

import functools
import struct
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import (kvr_block_norm, kvr_integer_product, kvr_linear_attention, kvr_linear_workspace, kvr_product_workspace)
from .serve import _current, _gpu, _no_gradient, _no_tangent, _refuse, _single, _status, _stream, _vector

DTYPE_CODES = {torch.bfloat16: 0, torch.float16: 1, torch.int8: 3, torch.float32: 4}
ACTIVATIONS = {"none": 0, "sigmoid": 1, "silu": 2}
HALVES = (torch.bfloat16, torch.float16)
PRODUCT_TYPES = (torch.int8, *HALVES)

# the structs of include/kvr.h, as struct packs them (tests compare the layouts)
NORM_RECORD = struct.Struct("<I6i2fi8Q5q")
PRODUCT_RECORD = struct.Struct("<I5i6Q3q")
LINEAR_RECORD = struct.Struct("<I7ifi5Q10q5Q")


class BlockNorm(NamedTuple):
    """What ``block_norm`` returns."""
    out: torch.Tensor                 # [tokens, dim]
    residual: Optional[torch.Tensor]  # [tokens, dim], None without a residual
    scale: Optional[torch.Tensor]     # [tokens] float32 of an 8-bit result, else None


def _matrix(where: str, name: str, t, dtypes, rows, dim, device):
    """data_ptr and row stride of a [rows, dim] tensor (None: of any number) whose rows are contiguous."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.device == device:
        shape = t.shape
        if len(shape) == 2 and (rows is None or shape[0] == rows) and (dim is None or shape[1] == dim):
            stride, one = t.stride()
            if shape[0] >> 31:
                _refuse(where, f"{name} has {shape[0]} rows (fewer than 2^31)")
            if one == 1 or shape[1] <= 1:
                return t.data_ptr(), stride
            _refuse(where, f"the elements of a row of {name} must be contiguous")
    _refuse(where, f"{name} must be [{'rows' if rows is None else rows}, {'dim' if dim is None else dim}] of "
                   f"{' or '.join(map(str, dtypes))} on {device}")


def _apart(where: str, name: str, t) -> None:
    """Refuses an output whose rows overlap."""
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        _refuse(where, f"the rows of {name} overlap")


def _overlap(n: int, step: int, m: int, each: int, size: int) -> bool:
    """Whether of n times m pieces of ``size`` elements, ``step`` and ``each`` apart, some overlap."""
    if m <= 1 or n <= 1:
        return (n > 1 and m == 1 and step < size) or (m > 1 and n == 1 and each < size)
    if step < each:
        n, step, m, each = m, each, n, step
    return each < size or step < (m - 1) * each + size


def block_norm(x: torch.Tensor, *, after: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
               activation: str = "none", residual: Optional[torch.Tensor] = None, residual_scale: float = 1.0,
               before: Optional[torch.Tensor] = None, eps: float = 1e-6, int8: bool = False, in_place: bool = False,
               out: Optional[torch.Tensor] = None) -> BlockNorm:
    """The norms behind and before a block, with its gate and the residual.

    ``x`` [tokens, dim], a block's result; ``after`` and ``before`` [dim]:
    weights of the norm of x, and of the norm of the new residual; ``gate``
    [tokens, dim] (expanded, where all tokens have the same) through
    ``activation`` ("none", "sigmoid", "silu"); ``residual`` [tokens, dim] of
    x's type or float32: ``residual + residual_scale * a`` takes its place.
    What is None is left out.  With ``int8`` the result is in 8-bit integers
    with a scale for each token (for ``integer_product``), else of x's type;
    with ``in_place`` the new residual is written over the old one.
    """
    where = "block_norm"
    device = _gpu(where, "x", x)
    if device.index != _current():
        with torch.cuda.device(device):
            return block_norm(x, after=after, gate=gate, activation=activation, residual=residual,
                              residual_scale=residual_scale, before=before, eps=eps, int8=int8, in_place=in_place,
                              out=out)
    dtype = x.dtype
    code = DTYPE_CODES.get(dtype, 3)
    if code > 1:
        _refuse(where, f"x of {dtype} is not supported (bfloat16, float16)")
    p_x, x0 = _matrix(where, "x", x, HALVES, None, None, device)
    tokens, dim = x.shape
    p_after = 0 if after is None else _vector(where, "after", after, dtype, dim, device)
    p_before = 0 if before is None else _vector(where, "before", before, dtype, dim, device)
    p_gate, g0 = (0, 0) if gate is None else _matrix(where, "gate", gate, (dtype,), tokens, dim, device)
    if activation not in ACTIVATIONS:
        _refuse(where, f"activation must be one of {', '.join(ACTIVATIONS)}")
    p_res = p_new = p_scale = res_code = r0 = n0 = 0
    new = scale = None
    if residual is not None:
        p_res, r0 = _matrix(where, "residual", residual, (dtype, torch.float32), tokens, dim, device)
        res_code = code if residual.dtype is dtype else 4
        if in_place:
            _apart(where, "residual", residual)
            new, p_new, n0 = residual, p_res, r0
        else:
            new = torch.empty_like(residual, memory_format=torch.contiguous_format)
            p_new, n0 = new.data_ptr(), dim
    elif in_place:
        _refuse(where, "in_place is for a residual")
    if x.requires_grad or (after is not None and after.requires_grad) or (gate is not None and gate.requires_grad) or \
            (residual is not None and residual.requires_grad) or (before is not None and before.requires_grad) or \
            (out is not None and out.requires_grad):
        _no_gradient(where)
    if forward_ad._current_level >= 0:
        _no_tangent(where, x, after, gate, residual, before, out)
    kind = torch.int8 if int8 else dtype
    if out is None:
        out = torch.empty_like(x, dtype=kind, memory_format=torch.contiguous_format)
        p_out, o0 = out.data_ptr(), dim
    else:
        p_out, o0 = _matrix(where, "out", out, (kind,), tokens, dim, device)
        _apart(where, "out", out)
    if int8:
        # (no kernel runs for rows without an element)
        scale = x.new_empty(tokens, dtype=torch.float32) if dim else x.new_zeros(tokens, dtype=torch.float32)
        p_scale = scale.data_ptr()
    if tokens and dim:
        kvr_block_norm(
            NORM_RECORD.pack(NORM_RECORD.size, code, res_code, 3 if int8 else code, tokens, dim,
                             ACTIVATIONS[activation], _single(where, "eps", eps),
                             _single(where, "residual_scale", residual_scale), 0, p_x, p_after, p_gate, p_res, p_before,
                             p_new, p_out, p_scale, x0, g0, r0, n0, o0),
            _stream(device.index))
    return BlockNorm(out, new, scale)


@functools.lru_cache(maxsize=4096)
def _product_bytes(code: int, out: int, tokens: int, dim: int, channels: int) -> int:
    """Workspace of kvr_integer_product, which these sizes decide; raises for what it refuses."""
    return kvr_product_workspace(PRODUCT_RECORD.pack(PRODUCT_RECORD.size, code, out, tokens, dim, channels, 0, 0, 0,
                                                     int(code == 3), 0, 0, 0, 0, 0))


def integer_product(x: torch.Tensor, weight: torch.Tensor, weight_scale: torch.Tensor, *,
                    x_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                    dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``x`` [tokens, dim] times ``weight`` [channels, dim] in 8-bit integers:
    [tokens, channels], element (t, c) the exact sum times ``x_scale[t]`` times
    ``weight_scale[c]``, plus ``bias[c]``.

    ``weight`` is int8; ``x`` is int8 with ``x_scale`` [tokens] float32, or
    bfloat16 or float16, and then brought to integers with the scale
    max |x[t]| / 127 in the call.  ``weight_scale`` and ``bias`` [channels]
    are float32.  ``dtype``: bfloat16, float16 or float32; by default x's, or
    bfloat16.  dim is a multiple of 16, and so are the strides of 8-bit rows.
    """
    where = "integer_product"
    device = _gpu(where, "x", x)
    if device.index != _current():
        with torch.cuda.device(device):
            return integer_product(x, weight, weight_scale, x_scale=x_scale, bias=bias, dtype=dtype, out=out)
    int8 = x.dtype is torch.int8
    p_x, x0 = _matrix(where, "x", x, PRODUCT_TYPES, None, None, device)
    tokens, dim = x.shape
    p_w, w0 = _matrix(where, "weight", weight, (torch.int8,), None, dim, device)
    channels = weight.shape[0]
    if int8 != (x_scale is not None):
        _refuse(where, "x_scale goes with x of torch.int8")
    f32 = torch.float32
    p_xs = _vector(where, "x_scale", x_scale, f32, tokens, device) if int8 else 0
    p_ws = _vector(where, "weight_scale", weight_scale, f32, channels, device)
    p_bias = 0 if bias is None else _vector(where, "bias", bias, f32, channels, device)
    if x.requires_grad or weight_scale.requires_grad or (int8 and x_scale.requires_grad) or \
            (bias is not None and bias.requires_grad) or (out is not None and out.requires_grad):
        _no_gradient(where)
    if forward_ad._current_level >= 0:
        _no_tangent(where, x, weight_scale, x_scale, bias, out)
    if dtype is None:
        dtype = out.dtype if out is not None else torch.bfloat16 if int8 else x.dtype
    code, to = DTYPE_CODES[x.dtype], DTYPE_CODES.get(dtype, 3)
    if to == 3:
        _refuse(where, f"a result of {dtype} is not supported (bfloat16, float16, float32)")
    if out is None:
        out = x.new_empty((tokens, channels), dtype=dtype)
        p_out, o0 = out.data_ptr(), channels
    else:
        p_out, o0 = _matrix(where, "out", out, (dtype,), tokens, channels, device)
        _apart(where, "out", out)
    nbytes = _product_bytes(code, to, tokens, dim, channels)
    p_work = 0
    if nbytes:
        ws = x.new_empty(nbytes, dtype=torch.uint8)
        p_work = ws.data_ptr()
    if tokens:
        kvr_integer_product(
            PRODUCT_RECORD.pack(PRODUCT_RECORD.size, code, to, tokens, dim, channels, p_x, p_w, p_out, p_xs, p_ws,
                                p_bias, x0, w0, o0),
            p_work, nbytes, _stream(device.index))
    return out


@functools.lru_cache(maxsize=65536)
def _linear_bytes(code: int, tokens: int, requests: int, heads: int, kv_heads: int, dim: int, ragged: bool) -> int:
    """Workspace of kvr_linear_attention, which these sizes decide; raises for what it refuses."""
    return kvr_linear_workspace(LINEAR_RECORD.pack(LINEAR_RECORD.size, code, tokens, requests, heads, kv_heads, dim, 1,
                                                   1.0, 0, *[0] * 16, int(ragged), 0, 0, 0))


def linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, state: torch.Tensor, log_decay: torch.Tensor,
                     read: torch.Tensor, write: Optional[torch.Tensor] = None,
                     row_start: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
                     out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Linear attention of the new tokens ``q`` [tokens, heads, dim], ``k`` and
    ``v`` [tokens, kv_heads, dim] with the decay exp(``log_decay``) [kv_heads]
    (float32, <= 0) of each key head.

    ``state`` [slots, kv_heads, dim, dim] float32 is the pool of states (of the
    last two dimensions the first belongs to the keys); request r begins with
    that of slot ``read[r]`` (-1: zero; several may read one, the state of
    their shared prefix) and leaves its last in slot ``write[r]`` (-1: nowhere;
    None: where it was read).  ``row_start`` [requests + 1] int32: first new
    token of each request (None: one each).  A slot that a request writes is
    not used by another one.  ``scale`` is dim ** -0.5 by default.  Returns
    ``out`` (like ``q`` unless given); ``status`` [1] int32 receives the
    KVR_DEV_* bits.  There is no gradient.  Without any request nothing is
    written.
    """
    where = "linear_attention"
    device = _gpu(where, "q", q)
    if device.index != _current():
        with torch.cuda.device(device):
            return linear_attention(q, k, v, state, log_decay, read, write, row_start, scale=scale, out=out,
                                    status=status)
    if q.requires_grad or k.requires_grad or v.requires_grad or state.requires_grad or log_decay.requires_grad:
        _no_gradient(where)
    if forward_ad._current_level >= 0:
        _no_tangent(where, q, k, v, state, log_decay, out)
    if q.dtype not in HALVES or q.dim() != 3:
        _refuse(where, "q must be [tokens, heads, dim] of torch.bfloat16 or torch.float16")
    tokens, heads, dim = q.shape
    if tokens * heads >> 31:
        _refuse(where, "tokens * heads must be below 2^31")
    for name, t in (("k", k), ("v", v)):
        if t.dtype is not q.dtype or t.device != device or t.dim() != 3 or t.shape != (tokens, k.shape[1], dim):
            _refuse(where, f"{name} must be [{tokens}, kv_heads, {dim}] of {q.dtype} on {device}, k like v")
    kv_heads = k.shape[1]
    if state.dtype is not torch.float32 or state.device != device or state.dim() != 4 or \
            state.shape[1:] != (kv_heads, dim, dim) or state.stride()[2:] != (dim, 1):
        _refuse(where, f"state must be [slots, {kv_heads}, {dim}, {dim}] of torch.float32 on {device}, the values of a "
                       "state contiguous")
    slots, i32 = state.shape[0], torch.int32
    s0, s1 = state.stride()[:2]
    if _overlap(slots, s0, kv_heads, s1, dim * dim):
        _refuse(where, "the states overlap")
    p_decay = _vector(where, "log_decay", log_decay, torch.float32, kv_heads, device)
    p_read = _vector(where, "read", read, i32, None, device)
    requests = read.shape[0]
    p_write = 0 if write is None else _vector(where, "write", write, i32, requests, device)
    p_rows = 0 if row_start is None else _vector(where, "row_start", row_start, i32, requests + 1, device)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != device:
        _refuse(where, "out must be like q")
    elif out.requires_grad:
        _no_gradient(where)
    q0, q1, q2 = q.stride()
    k0, k1, k2 = k.stride()
    v0, v1, v2 = v.stride()
    o0, o1, o2 = out.stride()
    if _overlap(tokens, o0, heads, o1, dim):
        _refuse(where, "the heads of out overlap")
    if q2 != 1 or k2 != 1 or v2 != 1 or o2 != 1:
        _refuse(where, "the elements of a head must be contiguous")
    code = DTYPE_CODES[q.dtype]
    args = LINEAR_RECORD.pack(LINEAR_RECORD.size, code, tokens, requests, heads, kv_heads, dim, slots,
                              dim ** -0.5 if scale is None else _single(where, "scale", scale), 0, q.data_ptr(),
                              k.data_ptr(), v.data_ptr(), out.data_ptr(), state.data_ptr(), q0, q1, k0, k1, v0, v1, o0,
                              o1, s0, s1, p_decay, p_rows, p_read, p_write, _status(where, status, device))
    if not requests:
        # the C call takes no empty batch; what it would refuse for one request is refused here too
        _linear_bytes(code, tokens, 1, heads, kv_heads, dim, True)
        if tokens and not p_rows:
            _refuse(where, "without row_start there is one token a request")
        return out
    nbytes = _linear_bytes(code, tokens, requests, heads, kv_heads, dim, bool(p_rows))
    ws = q.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    kvr_linear_attention(args, ws.data_ptr() if nbytes else 0, nbytes, _stream(device.index))
    return out
