"""Serving operators on torch tensors: page tables, cache store and
shared-prefix attention (``kvr_block_tables``, ``kvr_cache_store`` and
``kvr_shared_attention`` of include/kvr.h, which says what they compute).

The functions check what the C side cannot see (types, shapes, devices),
marshal the arguments and launch on torch's current stream of the tensors'
device.  They neither synchronise nor copy to the host; workspaces and outputs
come from torch's allocator.  Errors raise ``KvrError``.  They have no
gradients: a call whose result would need one is refused (call under
``torch.no_grad`` or ``torch.inference_mode``), and so is one whose result
would have a tangent.
"""
from __future__ import annotations

import functools
import struct
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import (KVR_EINVAL, KvrError, kvr_attention_workspace, kvr_block_tables, kvr_block_tables_workspace,
               kvr_cache_store, kvr_shared_attention)

DTYPE_CODES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}

# the structs of include/kvr.h, as struct packs them (tests compare the layouts)
TABLES_RECORD = struct.Struct("<I5iq11Q")
CACHE_RECORD = struct.Struct("<I5i2Q6q2Q")
STORE_RECORD = struct.Struct("<I3i2Q4q2Q")
ATTENTION_RECORD = struct.Struct("<I7ifi3Q4q6Q2qQ")


class BlockTables(NamedTuple):
    """What ``block_tables`` returns; the table and the ring are updated in place.

    ``row_start``, ``slots``, ``positions`` and (unless ``in_place``) ``held``
    are views of one allocation, which lives as long as one of them: clone
    what is kept beyond the step.
    """
    held: torch.Tensor       # [rows] int32: tokens of each row
    state: torch.Tensor      # [3] int64: ring head, ring tail, status bits
    row_start: torch.Tensor  # [rows + 1] int32: new tokens of the rows before
    slots: torch.Tensor      # [num_tokens] int32
    positions: torch.Tensor  # [num_tokens] int32


def _refuse(where: str, msg: str):
    raise KvrError(KVR_EINVAL, where, msg)


def _vector(where: str, name: str, t, dtype, n, device) -> int:
    """data_ptr of a contiguous vector of n values (None: of any number) on the device."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.is_contiguous() and \
            t.dim() == 1 and (n is None or t.shape[0] == n):
        return t.data_ptr()
    _refuse(where, f"{name} must be a contiguous vector" + ("" if n is None else f" of {n}") + f" of {dtype} on "
                   f"{device}")


def _table(where: str, name: str, t, rows, device):
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or t.device != device:
        _refuse(where, f"{name} must be a torch.int32 tensor on {device}")
    if t.dim() != 2 or t.shape[0] != rows:
        _refuse(where, f"{name} must be [{rows}, pages]")
    width = t.shape[1]
    stride, one = t.stride()
    if width > 1 and one != 1:
        _refuse(where, f"the pages of a row of {name} must be contiguous")
    if rows > 1 and stride < width:
        _refuse(where, f"the rows of {name} overlap")
    return t.data_ptr(), width, stride if stride > width else width


def _gpu(where: str, name: str, t) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(where, f"{name} must be a tensor on a GPU")
    return t.device


def _no_gradient(where: str) -> None:
    """Called where an argument requires one."""
    if torch.is_grad_enabled():
        _refuse(where, "there is no gradient: call under torch.no_grad(), or with detached tensors")


def _no_tangent(where: str, *tensors) -> None:
    """Called where forward mode has a level (``forward_ad._current_level`` >= 0)."""
    if torch._C._is_fwd_grad_enabled() and \
            any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        _refuse(where, "there is no tangent: call with the primal tensors")


_BEYOND = 2.0 ** 128 - 2.0 ** 103  # the first number that rounds past 32 bits


def _single(where: str, name: str, x) -> float:
    """A number that 32 bits hold (struct packs no others)."""
    if not -_BEYOND < x < _BEYOND:
        _refuse(where, f"{name} must be finite in 32 bits")
    return x


# of a device's index; of the current device
_stream, _current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


@functools.lru_cache(maxsize=4096)
def _tables_bytes(rows: int) -> int:
    """Workspace of kvr_block_tables, which only the number of rows decides."""
    return kvr_block_tables_workspace(TABLES_RECORD.pack(TABLES_RECORD.size, rows, 1, 1, 1, 0, 1, *[0] * 11))


@functools.lru_cache(maxsize=65536)
def _attention_bytes(code: int, kv_heads: int, dim: int, q_code: int, tokens: int, requests: int, groups: int,
                     heads: int) -> int:
    """Workspace of kvr_shared_attention, which these sizes decide; raises for what it refuses."""
    return kvr_attention_workspace(
        CACHE_RECORD.pack(CACHE_RECORD.size, code, 1, 1, kv_heads, dim, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0),
        ATTENTION_RECORD.pack(ATTENTION_RECORD.size, q_code, tokens, requests, groups, heads, 0, 0, 1.0, 0, 0, 0, 0, 0,
                              0, 0, 0, 1, 0, 0, 0, 0, 0, 0, 0, 0))


def block_tables(held: torch.Tensor, delta: torch.Tensor, table: torch.Tensor, ring: torch.Tensor,
                 state: torch.Tensor, page_size: int, num_tokens: int, *, base: Optional[torch.Tensor] = None,
                 in_place: bool = False) -> BlockTables:
    """Pages, slots and positions for rows that gain or lose tokens.

    ``held`` and ``delta`` [rows] int32: tokens of each row and their change;
    ``table`` [rows, width] int32; ``ring`` [pages of the pool] int32 with
    ``state`` [3] int64 = head, tail, status bits (``page_ring`` makes both);
    ``num_tokens``: an upper bound of the new tokens, the length of ``slots``
    and ``positions``; ``base`` [rows] int32: position of a row's first token.
    ``table`` and ``ring`` are updated in place, with ``in_place`` also
    ``held`` and ``state``, else new tensors are returned for these.  Without
    any row nothing changes.
    """
    where = "block_tables"
    device = _gpu(where, "held", held)
    if device.index != _current():
        with torch.cuda.device(device):
            return block_tables(held, delta, table, ring, state, page_size, num_tokens, base=base, in_place=in_place)
    rows = held.shape[0] if held.dim() == 1 else -1
    i32 = torch.int32
    p_held = _vector(where, "held", held, i32, None, device)
    p_delta = _vector(where, "delta", delta, i32, rows, device)
    p_base = 0 if base is None else _vector(where, "base", base, i32, rows, device)
    p_ring = _vector(where, "ring", ring, i32, None, device)
    p_state = _vector(where, "state", state, torch.int64, 3, device)
    p_table, width, stride = _table(where, "table", table, rows, device)
    if not 0 <= num_tokens < 1 << 31 or not 0 < page_size <= 1024:
        _refuse(where, "num_tokens must be in 0..2^31 - 1, page_size a power of two in 1..1024")
    if not rows:
        # the C call takes no empty batch; what it would refuse for one row is refused here too
        kvr_block_tables_workspace(TABLES_RECORD.pack(TABLES_RECORD.size, 1, max(1, width), page_size, ring.shape[0],
                                                      num_tokens, max(1, width), *[0] * 11))
        none = torch.full((2, num_tokens), -1, dtype=i32, device=device)
        return BlockTables(held if in_place else held.clone(), state if in_place else state.clone(),
                           torch.zeros(1, dtype=i32, device=device), none[0], none[1])
    nbytes = _tables_bytes(rows)
    # one allocation: the outputs, then the workspace on a 256-byte boundary
    outputs = 2 * rows + 1 + 2 * num_tokens
    work = outputs + 63 & -64
    whole = torch.empty(work + nbytes // 4, dtype=i32, device=device)
    held_out, row_start, slots, positions, _ = torch.split_with_sizes(
        whole, (rows, rows + 1, num_tokens, num_tokens, work - outputs + nbytes // 4))
    if in_place:
        held_out = held
    state_out = state if in_place else torch.empty_like(state)
    at = whole.data_ptr()
    kvr_block_tables(
        TABLES_RECORD.pack(TABLES_RECORD.size, rows, width, page_size, ring.shape[0], num_tokens, stride, p_held,
                           p_delta, p_base, p_table, p_ring, p_state, p_held if in_place else at,
                           state_out.data_ptr(), at + 4 * rows, at + 4 * (2 * rows + 1),
                           at + 4 * (2 * rows + 1 + num_tokens)),
        at + 4 * work, nbytes, _stream(device.index))
    return BlockTables(held_out, state_out, row_start, slots, positions)


def page_ring(num_pages: int, device="cuda"):
    """(ring, state) of a pool whose pages are all free."""
    return (torch.arange(num_pages, dtype=torch.int32, device=device),
            torch.tensor([0, num_pages, 0], dtype=torch.int64, device=device))


def _cache_args(where: str, kc: torch.Tensor, vc: torch.Tensor, ks, vs, device):
    """The packed kvr_cache of two [pages, page_size, kv_heads, dim] tensors."""
    code = DTYPE_CODES.get(kc.dtype, -1)
    if code < 0:
        _refuse(where, f"a cache of {kc.dtype} is not supported (bfloat16, float16, float8_e4m3fn)")
    if vc.dtype != kc.dtype or vc.device != device or kc.device != device:
        _refuse(where, f"k_cache and v_cache must have one type and be on {device}")
    if kc.dim() != 4 or vc.shape != kc.shape:
        _refuse(where, "k_cache and v_cache must be [pages, page_size, kv_heads, dim]")
    pages, page, heads, dim = kc.shape
    a0, a1, a2, a3 = kc.stride()
    b0, b1, b2, b3 = vc.stride()
    if a3 != 1 or b3 != 1:
        _refuse(where, "the elements of a head must be contiguous")
    p_ks = 0 if ks is None else _vector(where, "k_scale", ks, torch.float32, heads, device)
    p_vs = 0 if vs is None else _vector(where, "v_scale", vs, torch.float32, heads, device)
    if (p_ks and ks.requires_grad) or (p_vs and vs.requires_grad):
        _no_gradient(where)
    return CACHE_RECORD.pack(CACHE_RECORD.size, code, pages, page, heads, dim, kc.data_ptr(), vc.data_ptr(), a0, a1, a2,
                             b0, b1, b2, p_ks, p_vs)


def _status(where: str, status, device) -> int:
    return 0 if status is None else _vector(where, "status", status, torch.int32, 1, device)


def cache_store(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, slots: torch.Tensor, *,
                k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None) -> None:
    """Writes ``k`` and ``v`` [tokens, kv_heads, dim] into the slots [tokens]
    (int32) of ``k_cache`` and ``v_cache`` [pages, page_size, kv_heads, dim];
    tokens of a negative slot are skipped.  Any strides but the last
    dimension's: a cache with heads first is passed transposed.  A
    float8_e4m3fn cache holds x / scale[head]."""
    where = "cache_store"
    device = _gpu(where, "k", k)
    if device.index != _current():
        with torch.cuda.device(device):
            return cache_store(k, v, k_cache, v_cache, slots, k_scale=k_scale, v_scale=v_scale, status=status)
    if k.requires_grad or v.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
        _no_gradient(where)
    if forward_ad._current_level >= 0:
        _no_tangent(where, k, v, k_cache, v_cache, k_scale, v_scale)
    cache = _cache_args(where, k_cache, v_cache, k_scale, v_scale, device)
    shape = k.shape
    if k.dtype is not v.dtype or v.device != device or len(shape) != 3 or shape != v.shape or \
            shape[1:] != k_cache.shape[2:]:
        _refuse(where, f"k and v must be [tokens, {k_cache.shape[2]}, {k_cache.shape[3]}], of one type, on {device}")
    a0, a1, a2 = k.stride()
    b0, b1, b2 = v.stride()
    if a2 != 1 or b2 != 1:
        _refuse(where, "the elements of a head must be contiguous")
    p_slots = _vector(where, "slots", slots, torch.int32, shape[0], device)
    kvr_cache_store(cache, STORE_RECORD.pack(STORE_RECORD.size, DTYPE_CODES.get(k.dtype, -1), shape[0], 0, k.data_ptr(),
                                             v.data_ptr(), a0, a1, b0, b1, p_slots, _status(where, status, device)),
                    _stream(device.index))


def shared_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     row_start: Optional[torch.Tensor], table: torch.Tensor, length: torch.Tensor,
                     group_start: Optional[torch.Tensor] = None, prefix_table: Optional[torch.Tensor] = None,
                     prefix_length: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
                     k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the new tokens ``q`` [tokens, heads, dim] over their
    group's prefix and their request's own tokens up to themselves.

    ``row_start`` [requests + 1] int32: first new token of each request (None:
    one each); ``table`` [requests, width] int32 and ``length`` [requests]
    int32: pages and number of a request's own tokens, the new ones last;
    ``group_start`` [groups + 1], ``prefix_table`` [groups, width] and
    ``prefix_length`` [groups] int32: the requests of each group, and the
    pages and length of what they share (None: nothing is shared).  ``scale``
    is dim ** -0.5 by default.  Returns ``out`` (like ``q`` unless given);
    ``lse`` [tokens, heads] float32 receives the logarithms of the softmax
    sums, ``status`` [1] int32 the KVR_DEV_* bits.  There is no gradient.
    Without any request nothing is written.
    """
    where = "shared_attention"
    device = _gpu(where, "q", q)
    if device.index != _current():
        with torch.cuda.device(device):
            return shared_attention(q, k_cache, v_cache, row_start, table, length, group_start, prefix_table,
                                    prefix_length, scale=scale, k_scale=k_scale, v_scale=v_scale, out=out, lse=lse,
                                    status=status)
    if q.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
        _no_gradient(where)
    if forward_ad._current_level >= 0:
        _no_tangent(where, q, k_cache, v_cache, k_scale, v_scale, out)
    cache = _cache_args(where, k_cache, v_cache, k_scale, v_scale, device)
    _, _, kv_heads, dim = k_cache.shape
    if q.dim() != 3 or q.shape[2] != dim:
        _refuse(where, f"q must be [tokens, heads, {dim}]")
    tokens, heads, _ = q.shape
    i32 = torch.int32
    p_length = _vector(where, "length", length, i32, None, device)
    requests = length.shape[0]
    p_rows = 0 if row_start is None else _vector(where, "row_start", row_start, i32, requests + 1, device)
    p_table, width, stride = _table(where, "table", table, requests, device)
    groups = p_start = p_prefix = p_plen = pwidth = pstride = 0
    if prefix_length is not None or group_start is not None or prefix_table is not None:
        if prefix_length is None or group_start is None or prefix_table is None:
            _refuse(where, "group_start, prefix_table and prefix_length go together")
        p_plen = _vector(where, "prefix_length", prefix_length, i32, None, device)
        groups = prefix_length.shape[0]
        p_start = _vector(where, "group_start", group_start, i32, groups + 1, device)
        p_prefix, pwidth, pstride = _table(where, "prefix_table", prefix_table, groups, device)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != device:
        _refuse(where, "out must be like q")
    elif out.requires_grad:
        _no_gradient(where)
    q0, q1, q2 = q.stride()
    o0, o1, o2 = out.stride()
    if q2 != 1 or o2 != 1:
        _refuse(where, "the elements of a head must be contiguous")
    p_lse = 0
    if lse is not None:
        if lse.dtype != torch.float32 or lse.device != device or lse.shape != (tokens, heads) or \
                not lse.is_contiguous():
            _refuse(where, f"lse must be a contiguous float32 [{tokens}, {heads}] on {device}")
        p_lse = lse.data_ptr()
    code = DTYPE_CODES.get(q.dtype, -1)
    args = ATTENTION_RECORD.pack(ATTENTION_RECORD.size, code, tokens, requests, groups, heads, width, pwidth,
                                 dim ** -0.5 if scale is None else _single(where, "scale", scale), 0, q.data_ptr(),
                                 out.data_ptr(), p_lse, q0, q1, o0, o1, p_rows, p_length, p_table, p_start, p_prefix,
                                 p_plen, stride, pstride, _status(where, status, device))
    # (the C call takes no batch without requests)
    nbytes = _attention_bytes(DTYPE_CODES[k_cache.dtype], kv_heads, dim, code, tokens, requests or 1, groups, heads)
    if not requests:
        if tokens and not p_rows:
            _refuse(where, "without row_start there is one token a request")
        return out
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    kvr_shared_attention(cache, args, ws.data_ptr(), nbytes, _stream(device.index))
    return out


def check_status(where: str, bits: int) -> None:
    """Raises for the KVR_DEV_* bits of an operator's status (0: none)."""
    names = {1: "invalid lengths", 128: "the page ring holds too few pages", 256: "a row of a page table is too short",
             512: "a page number or slot outside the cache"}
    if bits:
        raise KvrError(KVR_EINVAL, where, ", ".join(t for b, t in names.items() if bits & b) or f"status {bits}")
