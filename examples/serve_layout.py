"""Serve a laid-out group of retrieval prompts from a paged prefix cache.

    python examples/serve_layout.py

The exact solver orders the passages of each request; the requests are then served in the layout's
order through one attention layer of random weights.  A request forks the row of the one before it
as far as their strings agree, so every node of the layout's trie is computed once: the tokens that
pass through the layer are the layout's cost.  After the prompts, all requests generate together: in
one call over their whole rows, and again with the prefix that all of them share attended once and
merged with their own suffixes.  At the end half of the requests leave and the cache is compacted.
"""

from __future__ import annotations

import os
import sys
from dataclasses import dataclass, field

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_13692_gb300 import instances, kv, mpt  # noqa: E402


class PagedCache:
    """Pages of one pool for several layers, with the rows that own them."""

    def __init__(self, layers, n_pages, page_size, kv_heads, head_dim, rows, width, dtype=torch.bfloat16):
        self.page_size = page_size
        self.pool = torch.empty((layers, n_pages, 2, page_size, kv_heads, head_dim), dtype=dtype, device="cuda")
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")

    @property
    def book(self):
        return self.table, self.lens, self.refs, self.page_size

    def pages(self, layer):
        return self.pool[layer, :, 0], self.pool[layer, :, 1]

    def fork(self, src, dst, keep):
        old, fresh, status = kv.mpt_kv_fork(*self.book, ints(src), ints(dst), ints(keep))
        kv.mpt_kv_copy_pages(self.pool, old, fresh)
        return status

    def extend(self, rows, more):
        return kv.mpt_kv_extend(*self.book, ints(rows), ints(more))

    def free(self, rows):
        return kv.mpt_kv_free(*self.book, ints(rows))

    def compact(self):
        old, fresh, status = kv.mpt_kv_compact(*self.book)
        kv.mpt_kv_copy_pages(self.pool, old, fresh)
        return status


def ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def offsets(lengths):
    return ints([0, *torch.tensor(lengths).cumsum(0).tolist()])


@dataclass
class Layer:
    """Random projections of token embeddings; the embedding of a token is drawn from its id."""

    heads: int
    kv_heads: int
    head_dim: int
    width: int = 256
    dtype: torch.dtype = torch.bfloat16
    weights: dict = field(default_factory=dict)

    def __post_init__(self):
        gen = torch.Generator(device="cuda").manual_seed(0)
        for name, n in (("q", self.heads), ("k", self.kv_heads), ("v", self.kv_heads)):
            w = torch.randn((self.width, n * self.head_dim), generator=gen, device="cuda") / self.width ** 0.5
            self.weights[name] = w.to(self.dtype)
        self.embedding = torch.randn((1 << 16, self.width), generator=gen, device="cuda").to(self.dtype)

    def project(self, tokens):
        x = self.embedding[tokens % (1 << 16)]
        return [(x @ self.weights[n]).view(len(tokens), -1, self.head_dim) for n in ("q", "k", "v")]


def prompt_tokens(chunks, weights):
    """The token ids of a string of passages: passage x has weights[x] tokens of its own."""
    return torch.cat([(torch.arange(int(weights[x])) + 977 * int(x)) for x in chunks]).cuda()


def common(a, b):
    n = 0
    while n < min(len(a), len(b)) and a[n] == b[n]:
        n += 1
    return n


def serve(m=12, steps=3, page_size=16, heads=16, kv_heads=4, head_dim=128, seed=0):
    """Returns what was computed: the layout's cost, the tokens prefilled, the prompts' outputs, each
    step's outputs by both ways, and the page counts before and after compaction."""
    inst = instances.zipf_small(m, 48, 5, 1.0, seed=seed)
    res = mpt.solve(inst.weights, inst.bits)
    strings = res.permutations()
    order = res.dfs_order.tolist()
    lengths = [int(sum(inst.weights[x] for x in s)) for s in strings]
    width = max(lengths) // page_size + 4
    cache = PagedCache(1, 2 * m * width, page_size, kv_heads, head_dim, m, width)
    layer = Layer(heads, kv_heads, head_dim)
    k_pages, v_pages = cache.pages(0)
    outputs, prefilled = {}, 0
    for at, r in enumerate(order):
        before = order[at - 1] if at else None
        shared = common(strings[before], strings[r]) if at else 0
        keep = int(sum(inst.weights[x] for x in strings[r][:shared]))
        if keep:
            cache.fork([before], [r], [keep])
        new = lengths[r] - keep
        prefilled += new
        if new:
            cache.extend([r], [new])
            q, k, v = layer.project(prompt_tokens(strings[r], inst.weights)[keep:])
            row = (cache.table[r:r + 1], offsets([new]), cache.lens[r:r + 1])
            kv.mpt_kv_write(k, v, k_pages, v_pages, *row)
            outputs[r] = (keep, kv.mpt_kv_attend(q, k_pages, v_pages, *row, max_q_len=new)[0])
    # all requests generate together
    prefix = strings[order[0]]
    for s in strings:
        prefix = prefix[:common(prefix, s)]
    shared = int(sum(inst.weights[x] for x in prefix)) // page_size * page_size  # whole pages of it
    both = []
    for step in range(steps):
        cache.extend(list(range(m)), [1] * m)
        q, k, v = layer.project(torch.arange(m, device="cuda") * 31 + 50_000 + step)
        row = (cache.table, offsets([1] * m), cache.lens)
        kv.mpt_kv_write(k, v, k_pages, v_pages, *row)
        whole = kv.mpt_kv_attend(q, k_pages, v_pages, *row, max_q_len=1)[0]
        # the shared prefix is one request of m tokens, each suffix starts after its pages
        first = order[0]
        parts = [kv.mpt_kv_attend(q, k_pages, v_pages, cache.table[first:first + 1], offsets([m]), ints([shared]),
                                  max_q_len=m, causal=False),
                 kv.mpt_kv_attend(q, k_pages, v_pages, cache.table[:, shared // page_size:], offsets([1] * m),
                                  cache.lens - shared, max_q_len=1)]
        both.append((whole, kv.mpt_kv_merge([p[0] for p in parts], [p[1] for p in parts])[0]))
    # half of the requests leave
    cache.free(list(range(0, m, 2)))
    stay = list(range(1, m, 2))
    q = layer.project(torch.arange(len(stay), device="cuda") + 40_000)[0]

    def look():
        return kv.mpt_kv_attend(q, k_pages, v_pages, cache.table[stay], offsets([1] * len(stay)), cache.lens[stay], max_q_len=1)[0]

    apart = look()
    live = int((cache.refs > 0).sum())
    last_before = int((cache.refs > 0).nonzero().max())
    cache.compact()
    together = look()
    kv.mpt_kv_check()
    return dict(cost=res.opt, prefilled=prefilled, strings=strings, weights=inst.weights, layer=layer, outputs=outputs, both=both,
                apart=apart, together=together, live=live, last_before=last_before,
                last_after=int((cache.refs > 0).nonzero().max()), tokens=sum(lengths), shared=shared)


if __name__ == "__main__":
    got = serve()
    print("prompt tokens %d, computed %d (the layout's cost: %d)" % (got["tokens"], got["prefilled"], got["cost"]))
    print("live pages %d, last one at %d before compaction, at %d after" % (got["live"], got["last_before"], got["last_after"]))
