"""Thin Python binding of ``include/mpt_kv.h``: a paged key/value cache for laid-out prompts.

``mpt.solve`` and its relatives order the chunks of prompts so that an exact-prefix cache is hit
most.  These operators serve such prompts: rows forked from a cached prefix, new keys and values
written into pages, attention of the new tokens over the cache, the merge of attention over parts
of the keys, and freeing and compacting pages.  Tensors are torch CUDA tensors, passed by address;
every step runs in the kernels of ``libmpt.so``.

Calls enqueue on ``stream`` (a raw stream address; default: torch's current stream) and return
without waiting.  What a call allocates (its outputs and workspace) belongs to that stream; inputs
that other streams write have to be ready in it, as for any torch operation.
"""

from __future__ import annotations

import contextlib
import ctypes
import math
from typing import Optional, Sequence

import torch

from . import mpt as _mpt

MPT_KV_BF16, MPT_KV_F16, MPT_KV_F32 = 0, 1, 2
MPT_KV_BAD_ROW, MPT_KV_NO_PAGES, MPT_KV_ROW_FULL = 1, 2, 4
_TYPES = {torch.bfloat16: MPT_KV_BF16, torch.float16: MPT_KV_F16, torch.float32: MPT_KV_F32}


class mpt_kv_cache(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3),
        ("type", ctypes.c_int32),
        ("n_pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("page_table", ctypes.c_void_p),
        ("table_stride", ctypes.c_int64),
        ("table_width", ctypes.c_int32),
        ("q_offsets", ctypes.c_void_p),
        ("kv_lens", ctypes.c_void_p),
    ]


class mpt_kv_book(ctypes.Structure):
    _fields_ = [
        ("table", ctypes.c_void_p),
        ("table_stride", ctypes.c_int64),
        ("width", ctypes.c_int32),
        ("rows", ctypes.c_int32),
        ("lens", ctypes.c_void_p),
        ("refs", ctypes.c_void_p),
        ("n_pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
    ]


@contextlib.contextmanager
def _on(tensor, stream):
    """The tensor's device, and `stream` as torch's current stream there, so that
    what the call allocates belongs to it; yields the stream's address."""
    if tensor.device.index == torch.cuda.current_device() and stream is None:
        yield torch.cuda.current_stream().cuda_stream
        return
    with torch.cuda.device(tensor.device):
        if stream is None:
            yield torch.cuda.current_stream().cuda_stream
        else:
            with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=tensor.device)):
                yield int(stream)


def _same_device(first, *others):
    for t in (first, *others):
        if not t.is_cuda or t.device != first.device:
            raise ValueError("every tensor must be on the same CUDA device")


def _ints(t, name: str, dims: int = 1):
    if t.dtype != torch.int32 or t.dim() != dims or (t.numel() > 0 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be a {dims}-d int32 tensor with contiguous rows")


def _cache(k_pages, v_pages, page_table, q_offsets, kv_lens) -> mpt_kv_cache:
    _same_device(k_pages, v_pages, page_table, q_offsets, kv_lens)
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype:
        raise ValueError("k_pages and v_pages must be [n_pages, page_size, kv_heads, head_dim] of one type")
    if k_pages.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("the cache must be bfloat16 or float16")
    if k_pages.stride(3) != 1 or v_pages.stride(3) != 1:
        raise ValueError("the elements of a head must be contiguous")
    _ints(page_table, "page_table", 2)
    _ints(q_offsets, "q_offsets")
    _ints(kv_lens, "kv_lens")
    batch = int(page_table.shape[0])
    if q_offsets.shape[0] != batch + 1 or kv_lens.shape[0] != batch:
        raise ValueError("q_offsets needs batch + 1 entries, kv_lens batch")
    n_pages, page_size, kv_heads, dim = k_pages.shape
    c = mpt_kv_cache(k_pages.data_ptr(), v_pages.data_ptr())
    c.k_stride[:] = k_pages.stride()[:3]
    c.v_stride[:] = v_pages.stride()[:3]
    c.type, c.n_pages, c.page_size, c.kv_heads, c.head_dim = _TYPES[k_pages.dtype], n_pages, page_size, kv_heads, dim
    c.batch, c.table_width = batch, page_table.shape[1]
    c.table_stride = max(page_table.stride(0), page_table.shape[1]) if batch < 2 else page_table.stride(0)
    c.page_table, c.q_offsets, c.kv_lens = page_table.data_ptr(), q_offsets.data_ptr(), kv_lens.data_ptr()
    return c


def _strides(t):
    return (ctypes.c_int64 * 2)(t.stride(0), t.stride(1))


_workspace_bytes: dict = {}


def mpt_kv_attend_workspace_bytes(head_dim: int) -> int:
    """Bytes of workspace of :func:`mpt_kv_attend` on the current device."""
    out = ctypes.c_size_t()
    _mpt._check(_mpt.load().mpt_kv_attend_workspace_bytes(int(head_dim), ctypes.byref(out)), "mpt_kv_attend_workspace_bytes")
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
    A row that sees no key gets out = 0, lse = -inf."""
    _same_device(q, k_pages)
    c = _cache(k_pages, v_pages, page_table, q_offsets, kv_lens)
    if q.dim() != 3 or q.dtype != k_pages.dtype or q.shape[2] != c.head_dim or (q.numel() > 0 and q.stride(2) != 1):
        raise ValueError("q must be [tokens, heads, head_dim] of the cache's type with contiguous heads")
    tokens, heads = int(q.shape[0]), int(q.shape[1])
    with _on(q, stream) as s:
        if out is None:
            # rows that belong to no request are not written
            out = torch.empty((tokens, heads, c.head_dim), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device)
        if out.shape != q.shape or out.dtype != q.dtype or (out.numel() > 0 and out.stride(2) != 1):
            raise ValueError("out must have q's shape and type, with contiguous heads")
        if lse.shape != (tokens, heads) or lse.dtype != torch.float32 or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32[tokens, heads]")
        _same_device(q, out, lse)
        if workspace is None:
            key = (q.device.index, c.head_dim)
            if key not in _workspace_bytes:
                _workspace_bytes[key] = mpt_kv_attend_workspace_bytes(c.head_dim)
            workspace = torch.empty(_workspace_bytes[key], dtype=torch.uint8, device=q.device)
        if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA uint8 tensor")
        _same_device(q, workspace)
        _mpt._check(_mpt.load().mpt_kv_attend(
            ctypes.byref(c), q.data_ptr(), _strides(q), tokens, heads, int(max_q_len), 1 if causal else 0,
            1.0 / math.sqrt(c.head_dim) if scale is None else float(scale), out.data_ptr(), _strides(out),
            lse.data_ptr(), workspace.data_ptr(), workspace.numel(), s), "mpt_kv_attend")
    return out, lse


def mpt_kv_merge(outs, lses, *, out=None, lse=None, stream: Optional[int] = None):
    """Merge attention results over disjoint sets of keys; returns (out, lse).

    outs: a sequence of [.., head_dim] tensors (or one tensor of them along its first axis), bf16,
    f16 or f32; lses: likewise, float32 [..].  Parts with lse = -inf have no part in a row."""
    outs, lses = list(outs), list(lses)
    if not outs or len(outs) != len(lses):
        raise ValueError("outs and lses must be non-empty and of one length")
    o = outs[0]
    _same_device(o, *outs, *lses)
    if o.dtype not in _TYPES or o.dim() < 1:
        raise ValueError("outs must be bfloat16, float16 or float32")
    for a, b in zip(outs, lses):
        if a.shape != o.shape or a.dtype != o.dtype or not a.is_contiguous():
            raise ValueError("outs must be contiguous and of one shape and type")
        if b.shape != o.shape[:-1] or b.dtype != torch.float32 or not b.is_contiguous():
            raise ValueError("lses must be contiguous float32 of outs' shape without the last axis")
    n, dim = len(outs), int(o.shape[-1])
    with _on(o, stream) as s:
        out = torch.empty_like(o) if out is None else out
        lse = torch.empty_like(lses[0]) if lse is None else lse
        _same_device(o, out, lse)
        if out.shape != o.shape or out.dtype != o.dtype or not out.is_contiguous():
            raise ValueError("out must be contiguous, of outs' shape and type")
        if lse.shape != o.shape[:-1] or lse.dtype != torch.float32 or not lse.is_contiguous():
            raise ValueError("lse must be contiguous float32 of lses' shape")
        ps = (ctypes.c_void_p * n)(*[t.data_ptr() for t in outs])
        pl = (ctypes.c_void_p * n)(*[t.data_ptr() for t in lses])
        _mpt._check(_mpt.load().mpt_kv_merge(ps, pl, n, lse.numel(), dim, _TYPES[o.dtype], out.data_ptr(),
                                             lse.data_ptr(), s), "mpt_kv_merge")
    return out, lse


def mpt_kv_write(k_new, v_new, k_pages, v_pages, page_table, q_offsets, kv_lens, *, stream: Optional[int] = None) -> None:
    """Write the new tokens' keys and values ([tokens, kv_heads, head_dim], the cache's type) into
    their pages: the last q_offsets[i+1] - q_offsets[i] of request i's kv_lens[i] positions."""
    c = _cache(k_pages, v_pages, page_table, q_offsets, kv_lens)
    _same_device(k_pages, k_new, v_new)
    for t in (k_new, v_new):
        if t.shape != (k_new.shape[0], c.kv_heads, c.head_dim) or t.dtype != k_pages.dtype or (t.numel() > 0 and t.stride(2) != 1):
            raise ValueError("k_new and v_new must be [tokens, kv_heads, head_dim] of the cache's type with contiguous heads")
    with _on(k_pages, stream) as s:
        _mpt._check(_mpt.load().mpt_kv_write(ctypes.byref(c), k_new.data_ptr(), _strides(k_new), v_new.data_ptr(),
                                             _strides(v_new), int(k_new.shape[0]), s), "mpt_kv_write")


# ---------------------------------------------------------------------------
# Bookkeeping of pages
# ---------------------------------------------------------------------------

def _book(table, lens, refs, page_size: int) -> mpt_kv_book:
    _same_device(table, lens, refs)
    _ints(table, "table", 2)
    _ints(lens, "lens")
    _ints(refs, "refs")
    if lens.shape[0] != table.shape[0]:
        raise ValueError("lens needs one entry per table row")
    rows, width = table.shape
    stride = max(table.stride(0), width) if rows < 2 else table.stride(0)
    return mpt_kv_book(table.data_ptr(), stride, width, rows, lens.data_ptr(), refs.data_ptr(), refs.shape[0], int(page_size))


def _lists(table, *lists):
    _same_device(table, *lists)
    for t in lists:
        _ints(t, "a list of rows or lengths")
        if t.shape != lists[0].shape:
            raise ValueError("the lists must be of one length")


def mpt_kv_pages_workspace_bytes(table, lens, refs, page_size: int) -> int:
    """Bytes of workspace of the bookkeeping calls."""
    b = _book(table, lens, refs, page_size)
    out = ctypes.c_size_t()
    _mpt._check(_mpt.load().mpt_kv_pages_workspace_bytes(ctypes.byref(b), ctypes.byref(out)), "mpt_kv_pages_workspace_bytes")
    return int(out.value)


def _pages_workspace(table, refs, workspace):
    if workspace is None:  # what mpt_kv_pages_workspace_bytes says: a header, one int per page and per row
        workspace = torch.empty(4 * (16 + refs.shape[0] + table.shape[0]), dtype=torch.uint8, device=table.device)
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA uint8 tensor")
    _same_device(table, workspace)
    return workspace


def mpt_kv_fork(table, lens, refs, page_size: int, src, dst, keep, *, workspace=None, stream: Optional[int] = None):
    """Row dst[j] (empty) gets the first keep[j] tokens of row src[j]: full pages shared, a part page
    copied to a fresh one.  Returns (old, fresh, status): int32[n] page pairs for
    :func:`mpt_kv_copy_pages` (-1 where nothing is to copy), and the device int32[2] status."""
    b = _book(table, lens, refs, page_size)
    _lists(table, src, dst, keep)
    n = int(src.shape[0])
    with _on(table, stream) as s:
        got = torch.empty(2 * n + 2, dtype=torch.int32, device=table.device)
        old, fresh, status = got[:n], got[n:2 * n], got[2 * n:]
        ws = _pages_workspace(table, refs, workspace)
        _mpt._check(_mpt.load().mpt_kv_fork(ctypes.byref(b), src.data_ptr(), dst.data_ptr(), keep.data_ptr(), n,
                                            old.data_ptr(), fresh.data_ptr(), status.data_ptr(), ws.data_ptr(),
                                            ws.numel(), s), "mpt_kv_fork")
    return old, fresh, status


def mpt_kv_extend(table, lens, refs, page_size: int, rows, more, *, workspace=None, stream: Optional[int] = None):
    """Row rows[j] grows by more[j] tokens onto fresh pages; returns the device int32[2] status."""
    b = _book(table, lens, refs, page_size)
    _lists(table, rows, more)
    with _on(table, stream) as s:
        status = torch.empty(2, dtype=torch.int32, device=table.device)
        ws = _pages_workspace(table, refs, workspace)
        _mpt._check(_mpt.load().mpt_kv_extend(ctypes.byref(b), rows.data_ptr(), more.data_ptr(), int(rows.shape[0]),
                                              status.data_ptr(), ws.data_ptr(), ws.numel(), s), "mpt_kv_extend")
    return status


def mpt_kv_free(table, lens, refs, page_size: int, rows, *, workspace=None, stream: Optional[int] = None):
    """The pages of the listed rows lose a reference, the rows are emptied; returns the device int32[2] status."""
    b = _book(table, lens, refs, page_size)
    _lists(table, rows)
    with _on(table, stream) as s:
        status = torch.empty(2, dtype=torch.int32, device=table.device)
        ws = _pages_workspace(table, refs, workspace)
        _mpt._check(_mpt.load().mpt_kv_free(ctypes.byref(b), rows.data_ptr(), int(rows.shape[0]), status.data_ptr(),
                                            ws.data_ptr(), ws.numel(), s), "mpt_kv_free")
    return status


def mpt_kv_compact(table, lens, refs, page_size: int, *, workspace=None, stream: Optional[int] = None):
    """Moves the live pages to the lowest ids; returns (old, fresh, status): int32[n_pages // 2] page
    pairs for :func:`mpt_kv_copy_pages` (the moves, then -1), and the device int32[2] status."""
    b = _book(table, lens, refs, page_size)
    n = int(refs.shape[0]) // 2
    with _on(table, stream) as s:
        got = torch.empty(2 * n + 2, dtype=torch.int32, device=table.device)
        old, fresh, status = got[:n], got[n:2 * n], got[2 * n:]
        ws = _pages_workspace(table, refs, workspace)
        _mpt._check(_mpt.load().mpt_kv_compact(ctypes.byref(b), old.data_ptr(), fresh.data_ptr(), status.data_ptr(),
                                               ws.data_ptr(), ws.numel(), s), "mpt_kv_compact")
    return old, fresh, status


def mpt_kv_copy_pages(pool, src, dst, *, stream: Optional[int] = None) -> None:
    """Copy pages src[j] -> dst[j] in every plane of ``pool`` ([planes, n_pages, ...], a page
    contiguous); pairs with an id out of range (-1) are skipped.  No dst may be a page of another pair."""
    _lists(src, src, dst)
    _same_device(pool, src)
    if pool.dim() < 3:
        raise ValueError("pool must be [planes, n_pages, ...]")
    page = pool[0, 0] if pool.shape[0] and pool.shape[1] else None
    if page is None or not page.is_contiguous():
        raise ValueError("the pool must not be empty and its pages must be contiguous")
    e = pool.element_size()
    planes, n_pages, size = int(pool.shape[0]), int(pool.shape[1]), page.numel() * e
    with _on(pool, stream) as s:
        _mpt._check(_mpt.load().mpt_kv_copy_pages(pool.data_ptr(), planes, pool.stride(0) * e if planes > 1 else 0,
                                                  n_pages, pool.stride(1) * e if n_pages > 1 else size, size,
                                                  src.data_ptr(), dst.data_ptr(), int(src.shape[0]), s),
                    "mpt_kv_copy_pages")


def mpt_kv_check(stream: Optional[int] = None) -> None:
    """Waits for the stream and raises if a kernel of this module gave up a bounded wait since the last check."""
    s = _mpt._default_stream_ptr() if stream is None else int(stream)
    _mpt._check(_mpt.load().mpt_kv_check(s), "mpt_kv_check")
