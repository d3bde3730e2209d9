"""Plain models of the paged-cache operators, for the tests: attention in 64 bits, request by request,
and the page bookkeeping as a host program over lists."""

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def attend(q, k_pages, v_pages, table, q_offsets, kv_lens, causal, scale):
    """(out, lse, bound of out, bound of lse) in float64 on q's device.

    The bounds follow from the formula: scores are 32-bit sums of d products (error at most d 2^-24
    scale sum |q k| each), which moves a probability by that much relatively; exp2 and the 32-bit sums
    over n keys add 2^-20 + n 2^-24; a probability is rounded to the type for the product with the
    values (unit roundoff u, or half the smallest subnormal), the result once more."""
    dev, u = q.device, UNIT[q.dtype]
    heads, dim = q.shape[1], q.shape[2]
    n_pages, page, kv_heads = k_pages.shape[:3]
    group = heads // kv_heads
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=dev)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    at, lens = q_offsets.tolist(), kv_lens.tolist()
    for i in range(len(lens)):
        n, kv = at[i + 1] - at[i], lens[i]
        if n <= 0:
            continue
        j = torch.arange(kv, device=dev)
        ids = table[i].long()[j // page] if kv else j
        there = (ids >= 0) & (ids < n_pages)
        j, ids = j[there], ids[there]
        if not len(j):
            continue
        limit = kv - n + torch.arange(n, device=dev) if causal else torch.full((n,), kv - 1, device=dev)
        hidden = j[None, :] > limit[:, None]
        for g in range(kv_heads):
            k = k_pages[ids, j % page, g].double()
            v = v_pages[ids, j % page, g].double()
            rows = slice(at[i], at[i + 1])
            for h in range(g * group, (g + 1) * group):
                x = q[rows, h].double()
                s = (x @ k.T) * scale
                s = torch.where(hidden, -math.inf, s)
                z = torch.logsumexp(s, 1)
                p = torch.where(hidden, 0.0, torch.exp(s - torch.where(torch.isinf(z), 0.0, z)[:, None]))
                vis = torch.where(hidden[:, :, None], 0.0, v[None]) if not bool(torch.isfinite(v).all()) else None
                o = p @ v if vis is None else torch.einsum("nk,nkd->nd", p, vis)
                a = p @ v.abs() if vis is None else torch.einsum("nk,nkd->nd", p, vis.abs())
                err = dim * 2.0 ** -24 * scale * (x.abs() @ torch.where(torch.isfinite(k), k, 0.0).abs().T).amax(1)
                err = err + 2.0 ** -20 + len(j) * 2.0 ** -24
                tiny = len(j) * 2.0 ** -25 * torch.where(torch.isfinite(v), v, 0.0).abs().max() if q.dtype == torch.float16 else 0.0
                out[rows, h], lse[rows, h] = o, z
                tol[rows, h] = u * o.abs() + (u + 2 * err[:, None]) * (1 + u) * a + tiny + 2.0 ** -24
                tol_lse[rows, h] = err + 2.0 ** -21 * z.abs() + 2.0 ** -20
    return out, lse, tol, tol_lse


class Book:
    """Table rows as lists of page ids, on the host."""

    def __init__(self, rows, width, n_pages, page):
        self.rows, self.width, self.page = rows, width, page
        self.table = [[] for _ in range(rows)]
        self.lens = [0] * rows
        self.refs = [0] * n_pages

    def free_ids(self):
        return [i for i, r in enumerate(self.refs) if r <= 0]

    def fork(self, src, dst, keep):
        free, pairs = iter(self.free_ids()), []
        new = []
        for s, n in zip(src, keep):
            full, part = divmod(n, self.page)
            row, pair = list(self.table[s][:full]), (-1, -1)
            for i in row:
                if i >= 0:
                    self.refs[i] += 1
            if part:
                old = self.table[s][full]
                if old >= 0:
                    pair = (old, next(free))
                    self.refs[pair[1]] = 1
                row.append(pair[1])
            new.append(row)
            pairs.append(pair)
        for d, row, n in zip(dst, new, keep):
            self.table[d], self.lens[d] = row, n
        return pairs

    def extend(self, rows, more):
        free = iter(self.free_ids())
        for r, n in zip(rows, more):
            have = -(-self.lens[r] // self.page)
            self.lens[r] += n
            for _ in range(-(-self.lens[r] // self.page) - have):
                i = next(free)
                self.refs[i] = 1
                self.table[r].append(i)

    def free(self, rows):
        for r in rows:
            for i in self.table[r]:
                if i >= 0:
                    self.refs[i] -= 1
            self.table[r], self.lens[r] = [], 0

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        src = [i for i in range(n, len(self.refs)) if self.refs[i] > 0]
        dst = [i for i in range(n) if self.refs[i] <= 0]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        self.table = [[to.get(i, i) for i in row] for row in self.table]
        return list(to.items())

    def tensors(self, device, stride=None):
        wide = torch.full((self.rows, stride or self.width), -7, dtype=torch.int32)
        wide[:, :self.width] = -1
        for r, row in enumerate(self.table):
            wide[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
        return (wide.to(device)[:, :self.width], torch.tensor(self.lens, dtype=torch.int32, device=device),
                torch.tensor(self.refs, dtype=torch.int32, device=device))
