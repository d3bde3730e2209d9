"""Plain models of the turned writes and of the cache in 4 bits, for the tests: the turn in 32-bit numpy
operations rounded one by one, codes in 64 bits, element by element of the page's layout."""

import math

import numpy as np
import torch

from tests import kv_model as M


def groups(dim):
    return -(-dim // 32)


def turned(x, table, rows, rot, adjacent):
    """x [tokens, heads, dim] float32, turned by rows `rows` of the table (float32 [.., rot]); rows that
    the table does not have leave it alone."""
    x = x.astype(np.float32).copy()
    ok = (rows >= 0) & (rows < len(table))
    t = table[np.clip(rows, 0, len(table) - 1)]
    c, s = t[:, None, :rot // 2], t[:, None, rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., :rot // 2], x[..., rot // 2:rot])
    one, two = a * c - b * s, b * c + a * s  # each operation rounded to 32 bits
    assert one.dtype == np.float32
    y = x.copy()
    if adjacent:
        y[..., 0:rot:2], y[..., 1:rot:2] = one, two
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = one, two
    return np.where(ok[:, None, None], y, x)


def codes(x):
    """x [.., dim] float32: codes [.., 32 n], step bytes and offset bytes [.., n]."""
    x = np.clip(np.where(np.isnan(x), np.float32(0), x), np.float32(-3360), np.float32(3360)).astype(np.float64)
    dim, n = x.shape[-1], groups(x.shape[-1])
    if dim < 32 * n:
        first = x[..., 32 * (n - 1):32 * (n - 1) + 1]
        x = np.concatenate([x, np.broadcast_to(first, (*x.shape[:-1], 32 * n - dim))], -1)
    x = x.reshape(*x.shape[:-1], n, 32)
    lo, hi = x.min(-1), x.max(-1)
    span = (hi - lo).astype(np.float32).astype(np.float64)  # 32-bit operations: rounded after each
    s = np.maximum(np.maximum((span / 15).astype(np.float32), (np.maximum(hi, -lo) / 120).astype(np.float32)), 2.0 ** -18).astype(np.float64)
    e = np.floor(np.log2(s)) - 3
    s = np.ceil(s * 2.0 ** -e) * 2.0 ** e
    z = np.rint((lo / s).astype(np.float32)).astype(np.float64)
    c = np.clip(np.rint((x / s[..., None]).astype(np.float32)).astype(np.float64) - z[..., None], 0, 15)
    mant, exp = np.frexp(16 * s)
    step = ((exp - 1 + 15) * 8 + (2 * mant - 1) * 8).astype(np.int64)
    return c.astype(np.int64).reshape(*c.shape[:-2], 32 * n), step, z.astype(np.int64) + 128


def put(pages, dim, page, slot, head, k, v):
    """Codes of one token's keys and values (float32 [dim]) into pages (uint8 numpy [n_pages, heads, bytes])."""
    n = groups(dim)
    tile = pages[page, head, slot // 8 * 288 * n:(slot // 8 + 1) * 288 * n]
    tok = slot % 8
    for value, x in ((0, k), (1, v)):
        c, step, off = codes(x)
        for piece in range(8 * n):
            h = sum(int(c[4 * piece + i]) << 4 * i for i in range(4))
            h = (h << 6 | h >> 10) & 0xFFFF
            at = 144 * n + tok // 2 * 32 * n + 4 * piece + 2 * (tok % 2) if value else tok * 16 * n + 2 * piece
            tile[at], tile[at + 1] = h & 255, h >> 8
        for g in range(n):
            if value:
                at = 272 * n + tok // 2 * 4 * n + 4 * g + tok % 2
                tile[at], tile[at + 2] = step[g], off[g]
            else:
                at = 128 * n + tok * 2 * n + 2 * g
                tile[at], tile[at + 1] = step[g], off[g]


def values(pages, dim):
    """What pages (uint8 tensor [n_pages, heads, bytes]) stand for: keys, values float32 [n_pages, page, heads, dim]."""
    n = groups(dim)
    n_pages, heads, size = pages.shape
    t = pages.reshape(n_pages, heads, size // (288 * n), 288 * n).long()
    dev = pages.device
    tok, e = torch.arange(8, device=dev)[:, None], torch.arange(dim, device=dev)[None]
    found = []
    for value in (0, 1):
        if value:
            at, mark, to_offset = 144 * n + tok // 2 * 32 * n + e // 4 * 4 + tok % 2 * 2, 272 * n + tok // 2 * 4 * n + e // 32 * 4 + tok % 2, 2
        else:
            at, mark, to_offset = tok * 16 * n + e // 4 * 2, 128 * n + tok * 2 * n + e // 32 * 2, 1
        half = t[..., at] | t[..., at + 1] << 8
        half = (half >> 6 | half << 10) & 0xFFFF
        c = half >> 4 * (e % 4) & 15
        step = t[..., mark].clamp(max=222)
        exp, frac = step >> 3, (step & 7).double() / 8
        s = torch.where(exp > 0, torch.exp2(exp.double() - 15) * (1 + frac), 2.0 ** -14 * frac) / 16
        x = (c + t[..., mark + to_offset] - 128).double() * s
        found.append(x.float().permute(0, 2, 3, 1, 4).reshape(n_pages, -1, heads, dim))
    return found


def attend(q, pages, table, q_offsets, kv_lens, causal, scale):
    """As kv_model.attend, with what the 4-bit kernels round besides: bf16 queries hold what is below 2^-14
    of their row's largest element to 2^-25 of it only, and probabilities below 2^-25 2^-11 of the reference,
    which the largest may be 2^5 below, may count for nothing."""
    k, v = values(pages, q.shape[2])
    out, lse, tol, tol_lse = M.attend(q, k, v, table, q_offsets, kv_lens, causal, scale)
    n = max(1, int(kv_lens.max())) if len(kv_lens) else 1
    x = q.double().abs().amax(2) * 2.0 ** -25 * scale * q.shape[2] * float(k.abs().max())
    tail = n * 2.0 ** -31 * float(v.abs().max())
    return out, lse, tol + 2 * x[..., None] * float(v.abs().max()) + tail, tol_lse + x


def angles(rows, rot):
    rate = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    a = np.arange(rows, dtype=np.float64)[:, None] * rate
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


assert math.isclose(float(values(torch.tensor([[[0] * 288]], dtype=torch.uint8), 32)[0][0, 0, 0, 0]), 0.0)
