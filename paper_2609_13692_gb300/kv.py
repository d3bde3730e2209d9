"""Thin Python binding of ``include/mpt_kv.h``: a paged key/value cache for laid-out prompts.

``mpt.solve`` and its relatives order the chunks of prompts so that an exact-prefix cache is hit
most.  These operators serve such prompts: rows forked from a cached prefix, new keys and values
written into pages, attention of the new tokens over the cache, the merge of attention over parts
of the keys, and freeing and compacting pages; keys and queries turned by their positions on the
way, and a cache that holds keys and values in 4 bits.  Tensors are torch CUDA tensors, passed by address;
every step runs in the kernels of ``libmpt.so``.

Calls enqueue on ``stream`` (a raw stream address; default: torch's current stream) and return
without waiting.  What a call allocates (its outputs and workspace) belongs to that stream; inputs
that other streams write have to be ready in it, as for any torch operation.

There is no backward pass: where gradients are recorded, a tensor that requires one is refused
(use ``torch.no_grad()`` or ``torch.inference_mode()``).
"""

from __future__ import annotations

import ctypes
import math
import struct
from typing import Optional

import torch

from . import mpt as _mpt

MPT_KV_BF16, MPT_KV_F16, MPT_KV_F32 = 0, 1, 2
MPT_KV_BAD_ROW, MPT_KV_NO_PAGES, MPT_KV_ROW_FULL = 1, 2, 4
_TYPES = {torch.bfloat16: MPT_KV_BF16, torch.float16: MPT_KV_F16, torch.float32: MPT_KV_F32}
_INT = torch.int32

# The structures of mpt_kv.h as packed bytes (native sizes and alignment): a
# call's host time is a good part of a small call, and filling a ctypes
# structure field by field costs as much as the call itself.
_CACHE = struct.Struct("@2P6q6iPqi2P")  # mpt_kv_cache
_BOOK = struct.Struct("@Pq2i2P2i")      # mpt_kv_book
_PAIR = struct.Struct("@2q")            # two strides
_TWO = struct.Struct("@2P")             # two addresses
_TURN = struct.Struct("@Pq4i3P4q")      # mpt_kv_turn
_CACHE4 = struct.Struct("@P2q5iPqi2P")  # mpt_kv4_cache

_load = _mpt.load
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_empty, _U8, _F32 = torch.empty, torch.uint8, torch.float32


def _run(index: int, stream: Optional[int], call, *args):
    """call(stream address, *args) with device `index` current and `stream` as torch's current
    stream there, so that what the call allocates belongs to it."""
    if stream is None and index == _current_device():
        return call(_raw_stream(index), *args)
    with torch.cuda.device(index):
        if stream is None:
            return call(_raw_stream(index), *args)
        with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=index)):
            return call(int(stream), *args)


def _device(first, *others) -> int:
    index = first.get_device()
    for t in others:
        if t.get_device() != index:
            index = -1
    if index < 0:
        raise ValueError("every tensor must be on the same CUDA device")
    return index


def _no_grad(*tensors):
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("there is no backward pass: call it under torch.no_grad(), or detach what requires gradients")


def _ints(t, name: str):
    if t.dtype is not _INT or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous 1-d int32 tensor")


def _table(t, name: str):
    """(rows, width, row stride) of a table of ints."""
    shape, strides = t.shape, t.stride()
    if t.dtype is not _INT or len(shape) != 2 or (strides[1] != 1 and shape[1] > 1):
        raise ValueError(f"{name} must be a 2-d int32 tensor with contiguous rows")
    rows, width = shape
    return rows, width, strides[0] if rows > 1 else max(width, 1)


def _cache(k_pages, v_pages, page_table, q_offsets, kv_lens):
    """The packed mpt_kv_cache, and (type, kv_heads, head_dim)."""
    shape, dtype = k_pages.shape, k_pages.dtype
    if len(shape) != 4 or shape != v_pages.shape or dtype is not v_pages.dtype:
        raise ValueError("k_pages and v_pages must be [n_pages, page_size, kv_heads, head_dim] of one type")
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise ValueError("the cache must be bfloat16 or float16")
    kp, ks, kh, ke = k_pages.stride()
    vp, vs, vh, ve = v_pages.stride()
    if ke != 1 or ve != 1:
        raise ValueError("the elements of a head must be contiguous")
    batch, width, stride = _table(page_table, "page_table")
    _ints(q_offsets, "q_offsets")
    _ints(kv_lens, "kv_lens")
    if q_offsets.shape[0] != batch + 1 or kv_lens.shape[0] != batch:
        raise ValueError("q_offsets needs batch + 1 entries, kv_lens batch")
    n_pages, page_size, kv_heads, dim = shape
    return _CACHE.pack(k_pages.data_ptr(), v_pages.data_ptr(), kp, ks, kh, vp, vs, vh, _TYPES[dtype], n_pages, page_size,
                       kv_heads, dim, batch, page_table.data_ptr(), stride, width, q_offsets.data_ptr(),
                       kv_lens.data_ptr()), dtype, kv_heads, dim


def _heads_strides(t, name: str) -> bytes:
    """The strides of a [tokens, heads, head_dim] tensor, the heads contiguous."""
    a, b, c = t.stride()
    if c != 1 and t.numel() > 0:
        raise ValueError(f"{name} must have contiguous heads")
    return _PAIR.pack(a, b)


def _check_workspace(workspace, index: int):
    if workspace.dtype is not _U8 or not workspace.is_contiguous() or workspace.get_device() != index:
        raise ValueError("workspace must be a contiguous CUDA uint8 tensor on the same device")


_workspace_bytes: dict = {}


def mpt_kv_attend_workspace_bytes(head_dim: int) -> int:
    """Bytes of workspace of :func:`mpt_kv_attend` on the current device."""
    out = ctypes.c_size_t()
    _mpt._check(_load().mpt_kv_attend_workspace_bytes(int(head_dim), ctypes.byref(out)), "mpt_kv_attend_workspace_bytes")
    return int(out.value)


def mpt_kv_attend(q, k_pages, v_pages, page_table, q_offsets, kv_lens, *, max_q_len: int = 0, causal: bool = True,
                  scale: Optional[float] = None, out=None, lse=None, workspace=None, stream: Optional[int] = None):
    """Attention of new tokens over a paged cache; returns (out, lse).

    q: [tokens, heads, head_dim]; k_pages, v_pages: [n_pages, page_size, kv_heads, head_dim], any
    strides with contiguous heads; page_table: int32[batch, width]; q_offsets: int32[batch + 1], the
    tokens of each request; kv_lens: int32[batch], its keys, the new tokens' last.  Token t of a
    request with n new tokens and L keys sees keys j <= L - n + t (causal) or all L.  max_q_len: the
    most new tokens of a request, where known (a hint).  scale: default 1 / sqrt(head_dim).
    out: [tokens, heads, head_dim] of q's type; lse: float32[tokens, heads], natural logarithm.
    A row that sees no key gets out = 0, lse = -inf; tokens of no request are not written."""
    index = _device(q, k_pages, v_pages, page_table, q_offsets, kv_lens)
    _no_grad(q, k_pages, v_pages, out, lse)
    cache, dtype, _, dim = _cache(k_pages, v_pages, page_table, q_offsets, kv_lens)
    shape = q.shape
    if len(shape) != 3 or q.dtype is not dtype or shape[2] != dim:
        raise ValueError("q must be [tokens, heads, head_dim] of the cache's type")
    strides = _heads_strides(q, "q")
    if out is not None:
        _device(q, out)
        if out.shape != shape or out.dtype is not dtype:
            raise ValueError("out must have q's shape and type")
        out = (out, _heads_strides(out, "out"))
    if lse is not None:
        _device(q, lse)
        if lse.shape != shape[:2] or lse.dtype is not _F32 or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32[tokens, heads]")
    if workspace is not None:
        _check_workspace(workspace, index)
    return _run(index, stream, _attend, index, cache, q, strides, shape, dtype, max_q_len, 1 if causal else 0,
                1.0 / math.sqrt(dim) if scale is None else scale, out, lse, workspace)


def _attend(s, index, cache, q, strides, shape, dtype, max_q_len, causal, scale, out, lse, workspace):
    (tokens, heads, dim), device = shape, q.device
    if out is None:
        out, out_strides = _empty(shape, dtype=dtype, device=device), _PAIR.pack(heads * dim, dim)
    else:
        out, out_strides = out
    if lse is None:
        lse = _empty((tokens, heads), dtype=_F32, device=device)
    if workspace is None:
        size = _workspace_bytes.get(index)
        if size is None:
            size = _workspace_bytes[index] = mpt_kv_attend_workspace_bytes(dim)
        workspace = _empty(size, dtype=_U8, device=device)
    else:
        size = workspace.numel()
    status = _load().mpt_kv_attend(cache, q.data_ptr(), strides, tokens, heads, max_q_len, causal, scale, out.data_ptr(),
                                   out_strides, lse.data_ptr(), workspace.data_ptr(), size, s)
    if status:
        _mpt._check(status, "mpt_kv_attend")
    return out, lse


def mpt_kv_merge(outs, lses, *, out=None, lse=None, stream: Optional[int] = None):
    """Merge attention results over disjoint sets of keys; returns (out, lse).

    outs: a sequence of [.., head_dim] tensors (or one tensor of them along its first axis), bf16,
    f16 or f32; lses: likewise, float32 [..].  Parts with lse = -inf have no part in a row."""
    n, po, shape, dtype, o = _parts(outs, "outs")
    nl, pl, rows, ldtype, z = _parts(lses, "lses")
    kind = _TYPES.get(dtype)
    if kind is None or not shape:
        raise ValueError("outs must be bfloat16, float16 or float32 with heads of a last axis")
    if n != nl or rows != shape[:-1] or ldtype is not _F32:
        raise ValueError("lses must be as many float32 tensors as outs, of their shape without the last axis")
    index = _device(o, z)
    _no_grad(out, lse)
    if out is not None:
        _device(o, out)
        if out.shape != shape or out.dtype is not dtype or not out.is_contiguous():
            raise ValueError("out must be contiguous, of outs' shape and type")
    if lse is not None:
        _device(o, lse)
        if lse.shape != rows or lse.dtype is not _F32 or not lse.is_contiguous():
            raise ValueError("lse must be contiguous float32 of lses' shape")
    return _run(index, stream, _merge, n, po, pl, shape, rows, dtype, kind, o.device, out, lse)


def _addresses(at: list) -> bytes:
    return struct.pack("@%dP" % len(at), *at)


def _parts(parts, name: str):
    """(number, packed addresses, shape, type, a tensor) of equal contiguous parts."""
    if isinstance(parts, torch.Tensor):
        _no_grad(parts)
        shape = parts.shape
        if not shape or shape[0] < 1 or not parts.is_contiguous():
            raise ValueError(f"{name} must be contiguous parts, one at least")
        n, at, step = shape[0], parts.data_ptr(), parts.stride(0) * parts.element_size()
        return n, _TWO.pack(at, at + step) if n == 2 else _addresses([at + i * step for i in range(n)]), shape[1:], parts.dtype, parts
    parts = list(parts)
    if not parts:
        raise ValueError(f"{name} must not be empty")
    first, n = parts[0], len(parts)
    _device(first, *parts)
    _no_grad(*parts)
    for t in parts:
        if t.shape != first.shape or t.dtype is not first.dtype or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous and of one shape and type")
    return n, _addresses([t.data_ptr() for t in parts]), first.shape, first.dtype, first


def _merge(s, n, po, pl, shape, rows, dtype, kind, device, out, lse):
    if out is None:
        out = _empty(shape, dtype=dtype, device=device)
    if lse is None:
        lse = _empty(rows, dtype=_F32, device=device)
    status = _load().mpt_kv_merge(po, pl, n, lse.numel(), shape[-1], kind, out.data_ptr(), lse.data_ptr(), s)
    if status:
        _mpt._check(status, "mpt_kv_merge")
    return out, lse


def mpt_kv_write(k_new, v_new, k_pages, v_pages, page_table, q_offsets, kv_lens, *, stream: Optional[int] = None) -> None:
    """Write the new tokens' keys and values ([tokens, kv_heads, head_dim], the cache's type) into
    their pages: the last q_offsets[i+1] - q_offsets[i] of request i's kv_lens[i] positions."""
    index = _device(k_pages, v_pages, page_table, q_offsets, kv_lens, k_new, v_new)
    _no_grad(k_new, v_new, k_pages, v_pages)
    cache, dtype, kv_heads, dim = _cache(k_pages, v_pages, page_table, q_offsets, kv_lens)
    shape = k_new.shape
    if len(shape) != 3 or shape[1] != kv_heads or shape[2] != dim or v_new.shape != shape or k_new.dtype is not dtype or v_new.dtype is not dtype:
        raise ValueError("k_new and v_new must be [tokens, kv_heads, head_dim] of the cache's type")
    _run(index, stream, _write, cache, k_new.data_ptr(), _heads_strides(k_new, "k_new"), v_new.data_ptr(),
         _heads_strides(v_new, "v_new"), shape[0])


def _write(s, *args):
    status = _load().mpt_kv_write(*args, s)
    if status:
        _mpt._check(status, "mpt_kv_write")


def _turn(rotation, positions, adjacent: bool, q, q_out, tokens: int, dim: int, dtype, index: int):
    """The packed mpt_kv_turn."""
    for t in (rotation, positions, q, q_out):
        if t is not None and t.get_device() != index:
            raise ValueError("every tensor must be on the same CUDA device")
    _no_grad(rotation, q, q_out)
    shape, strides = rotation.shape, rotation.stride()
    if len(shape) != 2 or rotation.dtype is not _F32 or (strides[1] != 1 and shape[1] > 1):
        raise ValueError("rotation must be a 2-d float32 tensor with contiguous rows: rot / 2 cosines, rot / 2 sines")
    rows, rot = shape
    if positions is not None:
        _ints(positions, "positions")
        if positions.shape[0] != tokens:
            raise ValueError("positions needs one entry per token")
    if q is None:
        if q_out is not None:
            raise ValueError("q_out without q")
        return _TURN.pack(rotation.data_ptr(), strides[0], rows, rot, 1 if adjacent else 0, 1,
                          0 if positions is None else positions.data_ptr(), 0, 0, 0, 0, 0, 0)
    qs = q.shape
    if len(qs) != 3 or qs[0] != tokens or qs[2] != dim or q.dtype is not dtype:
        raise ValueError("q must be [tokens, heads, head_dim] of k_new's type")
    if q_out.shape != qs or q_out.dtype is not dtype:
        raise ValueError("q_out must have q's shape and type")
    a, b, e = q.stride()
    c, d, f = q_out.stride()
    if (e != 1 or f != 1) and q.numel() > 0:
        raise ValueError("q and q_out must have contiguous heads")
    return _TURN.pack(rotation.data_ptr(), strides[0], rows, rot, 1 if adjacent else 0, qs[1],
                      0 if positions is None else positions.data_ptr(), q.data_ptr(), q_out.data_ptr(), a, b, c, d)


def mpt_kv_write_rotated(k_new, v_new, rotation, k_pages, v_pages, page_table, q_offsets, kv_lens, *, q=None, positions=None,
                         adjacent: bool = False, q_out=None, stream: Optional[int] = None):
    """:func:`mpt_kv_write` with the keys turned by their positions on the way, and the queries
    ``q`` ([tokens, heads, head_dim]) beside them; returns the turned queries (None without q).

    rotation: float32[positions, rot], of each position rot / 2 cosines, then rot / 2 sines.  The
    first rot elements of a head turn, i with i + rot / 2 (rot a multiple of 16) or, with
    ``adjacent``, 2 i with 2 i + 1 (of 8).  positions: int32[tokens], each token's row of
    ``rotation``; default: its position in the cache.  A token whose row is not there is dropped, its
    query is not turned.  q_out: where the turned queries go (q itself: in place, else memory that
    q, k_new and v_new have no part of); tokens of no request are not written."""
    index = _device(k_pages, v_pages, page_table, q_offsets, kv_lens, k_new, v_new)
    _no_grad(k_new, v_new, k_pages, v_pages)
    cache, dtype, kv_heads, dim = _cache(k_pages, v_pages, page_table, q_offsets, kv_lens)
    shape = k_new.shape
    if len(shape) != 3 or shape[1] != kv_heads or shape[2] != dim or v_new.shape != shape or k_new.dtype is not dtype or v_new.dtype is not dtype:
        raise ValueError("k_new and v_new must be [tokens, kv_heads, head_dim] of the cache's type")
    return _run(index, stream, _write_rotated, cache, k_new, v_new, rotation, positions, adjacent, q, q_out, index)


def _write_rotated(s, cache, k_new, v_new, rotation, positions, adjacent, q, q_out, index):
    tokens, _, dim = k_new.shape
    if q is not None and q_out is None:
        q_out = _empty(q.shape, dtype=q.dtype, device=q.device)
    turn = _turn(rotation, positions, adjacent, q, q_out, tokens, dim, k_new.dtype, index)
    status = _load().mpt_kv_write_rotated(cache, turn, k_new.data_ptr(), _heads_strides(k_new, "k_new"), v_new.data_ptr(),
                                          _heads_strides(v_new, "v_new"), tokens, s)
    if status:
        _mpt._check(status, "mpt_kv_write_rotated")
    return q_out


# ---------------------------------------------------------------------------
# A cache in 4 bits
# ---------------------------------------------------------------------------

def mpt_kv4_page_bytes(page_size: int, head_dim: int) -> int:
    """Bytes of one KV head of a page in 4 bits: pages are uint8[n_pages, kv_heads, these]."""
    out = ctypes.c_int64()
    _mpt._check(_load().mpt_kv4_page_bytes(int(page_size), int(head_dim), ctypes.byref(out)), "mpt_kv4_page_bytes")
    return int(out.value)


def _cache4(pages, page_table, q_offsets, kv_lens, dim: int) -> bytes:
    """The packed mpt_kv4_cache of heads of `dim` elements."""
    shape = pages.shape
    if len(shape) != 3 or pages.dtype is not _U8:
        raise ValueError("pages must be uint8[n_pages, kv_heads, page bytes]")
    a, b, c = pages.stride()
    if c != 1:
        raise ValueError("the bytes of a page's head must be contiguous")
    n_pages, kv_heads, size = shape
    tile = 288 * ((dim + 31) // 32)
    if dim < 1 or size % tile or size == 0:
        raise ValueError("a page's head must be page_size / 8 tiles of 288 bytes per 32 elements")
    batch, width, stride = _table(page_table, "page_table")
    _ints(q_offsets, "q_offsets")
    _ints(kv_lens, "kv_lens")
    if q_offsets.shape[0] != batch + 1 or kv_lens.shape[0] != batch:
        raise ValueError("q_offsets needs batch + 1 entries, kv_lens batch")
    return _CACHE4.pack(pages.data_ptr(), a, b, n_pages, size // tile * 8, kv_heads, dim, batch, page_table.data_ptr(), stride, width,
                        q_offsets.data_ptr(), kv_lens.data_ptr())


def mpt_kv4_write(k_new, v_new, pages, page_table, q_offsets, kv_lens, *, rotation=None, q=None, positions=None,
                  adjacent: bool = False, q_out=None, stream: Optional[int] = None):
    """Write the new tokens' keys and values ([tokens, kv_heads, head_dim], bf16 or f16) as 4-bit
    codes into ``pages`` (uint8[n_pages, kv_heads, :func:`mpt_kv4_page_bytes`]).  With ``rotation``
    the keys are turned first, and ``q`` beside them, as by :func:`mpt_kv_write_rotated`; returns the
    turned queries (None without q)."""
    index = _device(pages, page_table, q_offsets, kv_lens, k_new, v_new)
    _no_grad(k_new, v_new)
    shape, dtype = k_new.shape, k_new.dtype
    if len(shape) != 3 or v_new.shape != shape or v_new.dtype is not dtype or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise ValueError("k_new and v_new must be [tokens, kv_heads, head_dim], bfloat16 or float16")
    cache = _cache4(pages, page_table, q_offsets, kv_lens, shape[2])
    if shape[1] != pages.shape[1]:
        raise ValueError("k_new and v_new must have the KV heads of pages")
    if rotation is None and (q is not None or positions is not None or q_out is not None):
        raise ValueError("q, positions and q_out go with a rotation")
    return _run(index, stream, _write4, cache, k_new, v_new, rotation, positions, adjacent, q, q_out, index)


def _write4(s, cache, k_new, v_new, rotation, positions, adjacent, q, q_out, index):
    tokens, _, dim = k_new.shape
    turn = None
    if rotation is not None:
        if q is not None and q_out is None:
            q_out = _empty(q.shape, dtype=q.dtype, device=q.device)
        turn = _turn(rotation, positions, adjacent, q, q_out, tokens, dim, k_new.dtype, index)
    status = _load().mpt_kv4_write(cache, turn, _TYPES[k_new.dtype], k_new.data_ptr(), _heads_strides(k_new, "k_new"),
                                   v_new.data_ptr(), _heads_strides(v_new, "v_new"), tokens, s)
    if status:
        _mpt._check(status, "mpt_kv4_write")
    return q_out


def mpt_kv4_read(pages, page_table, q_offsets, kv_lens, tokens: int, head_dim: int, *, dtype=torch.bfloat16, k_out=None, v_out=None,
                 stream: Optional[int] = None):
    """What the new tokens' codes stand for, in bf16, f16 or f32; returns (keys, values), each
    [tokens, kv_heads, head_dim] (k_out, v_out: where they go, without overlap).  0 for tokens that
    the cache has no place for; tokens of no request are not written."""
    index = _device(pages, page_table, q_offsets, kv_lens)
    cache = _cache4(pages, page_table, q_offsets, kv_lens, int(head_dim))
    kind = _TYPES.get(dtype)
    if kind is None:
        raise ValueError("dtype must be bfloat16, float16 or float32")
    shape = (int(tokens), pages.shape[1], int(head_dim))
    for t in (k_out, v_out):
        if t is not None:
            _device(pages, t)
            if t.shape != shape or t.dtype is not dtype:
                raise ValueError("k_out and v_out must be [tokens, kv_heads, head_dim] of dtype")
    _no_grad(k_out, v_out)
    return _run(index, stream, _read4, cache, kind, shape, dtype, pages.device, k_out, v_out)


def _read4(s, cache, kind, shape, dtype, device, k_out, v_out):
    if k_out is None:
        k_out = _empty(shape, dtype=dtype, device=device)
    if v_out is None:
        v_out = _empty(shape, dtype=dtype, device=device)
    status = _load().mpt_kv4_read(cache, kind, k_out.data_ptr(), _heads_strides(k_out, "k_out"), v_out.data_ptr(),
                                  _heads_strides(v_out, "v_out"), shape[0], s)
    if status:
        _mpt._check(status, "mpt_kv4_read")
    return k_out, v_out


_workspace4_bytes: dict = {}


def mpt_kv4_attend_workspace_bytes() -> int:
    """Bytes of workspace of :func:`mpt_kv4_attend` on the current device."""
    out = ctypes.c_size_t()
    _mpt._check(_load().mpt_kv4_attend_workspace_bytes(ctypes.byref(out)), "mpt_kv4_attend_workspace_bytes")
    return int(out.value)


def mpt_kv4_attend(q, pages, page_table, q_offsets, kv_lens, *, max_q_len: int = 0, causal: bool = True,
                   scale: Optional[float] = None, out=None, lse=None, workspace=None, stream: Optional[int] = None):
    """:func:`mpt_kv_attend` over a cache in 4 bits (:func:`mpt_kv4_write`); returns (out, lse).

    q: [tokens, heads, head_dim], bf16 or f16; pages: uint8[n_pages, kv_heads, page bytes].  Its
    other arguments, what rows without keys get and what is not written are those of
    :func:`mpt_kv_attend`."""
    index = _device(q, pages, page_table, q_offsets, kv_lens)
    _no_grad(q, out, lse)
    shape, dtype = q.shape, q.dtype
    if len(shape) != 3 or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise ValueError("q must be [tokens, heads, head_dim], bfloat16 or float16")
    dim = shape[2]
    cache = _cache4(pages, page_table, q_offsets, kv_lens, dim)
    strides = _heads_strides(q, "q")
    if out is not None:
        _device(q, out)
        if out.shape != shape or out.dtype is not dtype:
            raise ValueError("out must have q's shape and type")
        out = (out, _heads_strides(out, "out"))
    if lse is not None:
        _device(q, lse)
        if lse.shape != shape[:2] or lse.dtype is not _F32 or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32[tokens, heads]")
    if workspace is not None:
        _check_workspace(workspace, index)
    return _run(index, stream, _attend4, index, cache, q, strides, shape, dtype, max_q_len, 1 if causal else 0,
                1.0 / math.sqrt(dim) if scale is None else scale, out, lse, workspace)


def _attend4(s, index, cache, q, strides, shape, dtype, max_q_len, causal, scale, out, lse, workspace):
    (tokens, heads, dim), device = shape, q.device
    if out is None:
        out, out_strides = _empty(shape, dtype=dtype, device=device), _PAIR.pack(heads * dim, dim)
    else:
        out, out_strides = out
    if lse is None:
        lse = _empty((tokens, heads), dtype=_F32, device=device)
    if workspace is None:
        size = _workspace4_bytes.get(index)
        if size is None:
            size = _workspace4_bytes[index] = mpt_kv4_attend_workspace_bytes()
        workspace = _empty(size, dtype=_U8, device=device)
    else:
        size = workspace.numel()
    status = _load().mpt_kv4_attend(cache, _TYPES[dtype], q.data_ptr(), strides, tokens, heads, max_q_len, causal, scale,
                                    out.data_ptr(), out_strides, lse.data_ptr(), workspace.data_ptr(), size, s)
    if status:
        _mpt._check(status, "mpt_kv4_attend")
    return out, lse


# ---------------------------------------------------------------------------
# Bookkeeping of pages
# ---------------------------------------------------------------------------

def _book(table, lens, refs, page_size: int, *lists):
    """The packed mpt_kv_book, the device, the number of pages and the length of the lists."""
    index = _device(table, lens, refs, *lists)
    rows, width, stride = _table(table, "table")
    _ints(lens, "lens")
    _ints(refs, "refs")
    if len(lens) != rows:
        raise ValueError("lens needs one entry per table row")
    n = None
    for t in lists:
        _ints(t, "a list of rows or lengths")
        if n is None:
            n = len(t)
        elif len(t) != n:
            raise ValueError("the lists must be of one length")
    n_pages = len(refs)
    return _BOOK.pack(table.data_ptr(), stride, width, rows, lens.data_ptr(), refs.data_ptr(), n_pages,
                      int(page_size)), index, n_pages, n


def mpt_kv_fork(table, lens, refs, page_size: int, src, dst, keep, *, stream: Optional[int] = None):
    """Row dst[j] (empty) gets the first keep[j] tokens of row src[j]: full pages shared, a part page
    copied to a fresh one.  Returns (old, fresh, status): int32[n] page pairs for
    :func:`mpt_kv_copy_pages` (-1 where nothing is to copy), and the device int32[2] status."""
    book, index, n_pages, n = _book(table, lens, refs, page_size, src, dst, keep)
    return _run(index, stream, _fork, book, n, table.device, src, dst, keep)


def _fork(s, book, n, device, src, dst, keep):
    old, fresh = _empty(n, dtype=_INT, device=device), _empty(n, dtype=_INT, device=device)
    status = _empty(2, dtype=_INT, device=device)
    st = _load().mpt_kv_fork(book, src.data_ptr(), dst.data_ptr(), keep.data_ptr(), n, old.data_ptr(), fresh.data_ptr(),
                             status.data_ptr(), s)
    if st:
        _mpt._check(st, "mpt_kv_fork")
    return old, fresh, status


def mpt_kv_extend(table, lens, refs, page_size: int, rows, more, *, stream: Optional[int] = None):
    """Row rows[j] grows by more[j] tokens onto fresh pages; returns the device int32[2] status."""
    book, index, _, n = _book(table, lens, refs, page_size, rows, more)
    return _run(index, stream, _extend, book, n, table.device, rows, more)


def _extend(s, book, n, device, rows, more):
    status = _empty(2, dtype=_INT, device=device)
    st = _load().mpt_kv_extend(book, rows.data_ptr(), more.data_ptr(), n, status.data_ptr(), s)
    if st:
        _mpt._check(st, "mpt_kv_extend")
    return status


def mpt_kv_free(table, lens, refs, page_size: int, rows, *, stream: Optional[int] = None):
    """The pages of the listed rows lose a reference, the rows are emptied; returns the device int32[2] status."""
    book, index, _, n = _book(table, lens, refs, page_size, rows)
    return _run(index, stream, _free, book, n, table.device, rows)


def _free(s, book, n, device, rows):
    status = _empty(2, dtype=_INT, device=device)
    st = _load().mpt_kv_free(book, rows.data_ptr(), n, status.data_ptr(), s)
    if st:
        _mpt._check(st, "mpt_kv_free")
    return status


def mpt_kv_compact(table, lens, refs, page_size: int, *, stream: Optional[int] = None):
    """Moves the live pages to the lowest ids; returns (old, fresh, status): int32[n_pages // 2] page
    pairs for :func:`mpt_kv_copy_pages` (the moves, then -1), and the device int32[2] status."""
    book, index, n_pages, _ = _book(table, lens, refs, page_size)
    return _run(index, stream, _compact, book, n_pages // 2, table.device)


def _compact(s, book, n, device):
    old, fresh = _empty(n, dtype=_INT, device=device), _empty(n, dtype=_INT, device=device)
    status = _empty(2, dtype=_INT, device=device)
    st = _load().mpt_kv_compact(book, old.data_ptr(), fresh.data_ptr(), status.data_ptr(), s)
    if st:
        _mpt._check(st, "mpt_kv_compact")
    return old, fresh, status


def mpt_kv_copy_pages(pool, src, dst, *, stream: Optional[int] = None) -> None:
    """Copy pages src[j] -> dst[j] in every plane of ``pool`` ([planes, n_pages, ...], a page
    contiguous); pairs with an id out of range (-1) are skipped.  No dst may be a page of another pair."""
    index = _device(pool, src, dst)
    _no_grad(pool)
    _ints(src, "src")
    _ints(dst, "dst")
    if src.shape != dst.shape:
        raise ValueError("the lists must be of one length")
    shape, strides = pool.shape, pool.stride()
    if len(shape) < 3 or 0 in shape:
        raise ValueError("pool must be [planes, n_pages, ...] and not empty")
    size = 1
    for n, step in zip(shape[:1:-1], strides[:1:-1]):
        if n > 1 and step != size:
            raise ValueError("a page of the pool must be contiguous")
        size *= n
    e = pool.element_size()
    _run(index, stream, _copy_pages, pool, shape[0], strides[0] * e if shape[0] > 1 else 0, shape[1],
         (strides[1] if shape[1] > 1 else size) * e, size * e, src, dst)


def _copy_pages(s, pool, planes, plane_stride, n_pages, page_stride, page_bytes, src, dst):
    st = _load().mpt_kv_copy_pages(pool.data_ptr(), planes, plane_stride, n_pages, page_stride, page_bytes, src.data_ptr(),
                                       dst.data_ptr(), src.shape[0], s)
    if st:
        _mpt._check(st, "mpt_kv_copy_pages")


def mpt_kv_check(stream: Optional[int] = None) -> None:
    """Waits for the stream and raises if a kernel of this module, on any stream of the current device, gave up a
    bounded wait (or, in the bounds-checked build, left out an access) that no check has told of."""
    s = _mpt._default_stream_ptr() if stream is None else int(stream)
    _mpt._check(_load().mpt_kv_check(s), "mpt_kv_check")
