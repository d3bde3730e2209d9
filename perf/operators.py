"""Cases for measuring the paged-cache operators: what a program that serves laid-out prompts does with them.

After the layout, such a program keeps the prompts' keys and values in pages, forks a cached prefix for
each request that extends it, writes the new tokens, attends over the cache (a chunk of new tokens, or one
token per request), merges what shared prefixes and own suffixes gave, and frees and compacts pages.
Lengths go with the repository's workloads: groups of 12 to 28 requests of 5 to 20 passages of about 150
tokens, and long streams.  All inputs are synthetic, drawn from the seed.
"""

import math
import random

import torch

own = False  # False: the operators in elementary torch operations, in 32 bits; True: the framework's kernels

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

LISTED = [
    # One request's next token over a prompt of a few passages: nothing but latency.
    dict(name="decode_one", kind="attend", batch=1, q_lo=1, q_hi=1, kv_lo=777, kv_hi=777, heads=32, kv_heads=8,
         dim=128, page=16, dtype="bf16", order="token", causal=True, holes=False),
    # The benchmark's group of 28 requests, each at its next token over its prompt of 20 passages.
    dict(name="decode_m28", kind="attend", batch=28, q_lo=1, q_hi=1, kv_lo=2000, kv_hi=6000, heads=32, kv_heads=8,
         dim=128, page=16, dtype="bf16", order="token", causal=True, holes=False),
    # Few requests over very long contexts (a million-passage workload's deep retrieval), 64-token pages kept head by head.
    dict(name="decode_long", kind="attend", batch=3, q_lo=1, q_hi=1, kv_lo=100_001, kv_hi=131_072, heads=64,
         kv_heads=8, dim=128, page=64, dtype="f16", order="head", causal=True, holes=False),
    # 28 requests in one step of a continuous batch: some at one token, others with up to 700 new ones; odd head size.
    dict(name="chunk_ragged", kind="attend", batch=28, q_lo=1, q_hi=700, kv_lo=700, kv_hi=6000, heads=24, kv_heads=8,
         dim=96, page=32, dtype="f16", order="token", causal=True, holes=True),
    # A long prompt's chunk: 4,096 new tokens over 16,384 cached ones.
    dict(name="chunk_long", kind="attend", batch=1, q_lo=4096, q_hi=4096, kv_lo=20_480, kv_hi=20_480, heads=32,
         kv_heads=8, dim=128, page=16, dtype="bf16", order="token", causal=True, holes=False),
    # The next tokens of 28 requests over the prefix that they share, which is read once for all of them.
    dict(name="prefix_shared", kind="attend", batch=1, q_lo=28, q_hi=28, kv_lo=20_001, kv_hi=20_001, heads=32,
         kv_heads=8, dim=128, page=16, dtype="bf16", order="token", causal=False, holes=False),
    # Shared prefix and own suffix of 28 next tokens, brought together.
    dict(name="merge_m28", kind="merge", parts=2, tokens=28, heads=32, dim=128, dtype="bf16", empty=True),
    # Four trie levels of a long chunk.
    dict(name="merge_8192", kind="merge", parts=4, tokens=8192, heads=32, dim=128, dtype="bf16", empty=False),
    # One new token for each of 28 requests.
    dict(name="write_m28", kind="write", batch=28, q_lo=1, q_hi=1, kv_lo=2000, kv_hi=6000, kv_heads=8, dim=128,
         page=16, dtype="bf16", order="token"),
    # The new tokens of a prefill step.
    dict(name="write_prefill", kind="write", batch=28, q_lo=300, q_hi=2100, kv_lo=2200, kv_hi=4000, kv_heads=8,
         dim=128, page=16, dtype="bf16", order="token"),
    # 28 requests of a group forked from their common prefixes and grown by a passage.
    dict(name="pages_fork_m28", kind="fork", rows=64, table=512, forks=28, planes=16, pages=4096, page=16, kv_heads=8,
         dim=128, dtype="bf16", fill=0.6),
    # Half of a worn pool's requests end; what is left is brought together at the front.
    dict(name="pages_compact", kind="compact", rows=1000, table=256, forks=500, planes=4, pages=65_536, page=16,
         kv_heads=4, dim=64, dtype="bf16", fill=0.9),
]


def listed():
    return [dict(c) for c in LISTED]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST_FLOPS = 1.0e12   # of a drawn attention (chunk_long: 1.2e12)
MOST_BYTES = 1.2e9    # (decode_long: 1.4e9)
MOST_SCORES = 4.0e9   # entries of the plain form's score matrix, padding among them


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend", "attend", "merge", "write", "fork", "compact"])
    dtype = rng.choice(["bf16", "f16"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    dim = rng.choice([64, 128, 128, 128, 96, 80, 256])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    order = rng.choice(["token", "head"])
    if kind == "merge":
        c = dict(kind=kind, parts=rng.randint(2, 8), tokens=_log_int(rng, 1, 8192), heads=kv_heads * rng.choice([1, 2, 4]),
                 dim=dim, dtype=rng.choice(["bf16", "f16", "f32"]), empty=rng.random() < 0.5)
        while c["parts"] * c["tokens"] * c["heads"] * dim > 1.2e8:
            c["tokens"] = c["tokens"] * 2 // 3
        return c
    if kind == "write":
        lo = _log_int(rng, 1, 1000)
        c = dict(kind=kind, batch=_log_int(rng, 1, 256), q_lo=lo, q_hi=_log_int(rng, lo, 2 * lo + 1), kv_lo=2 * lo + 1,
                 kv_hi=_log_int(rng, 2 * lo + 1, 6000), kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, order=order)
        while work(c)["bytes"] > 2.0e8:
            c["batch"] = c["batch"] * 2 // 3
        return c
    if kind == "fork":
        rows = _log_int(rng, 16, 1000)
        forks = rng.randint(1, rows // 2)
        pages = _log_int(rng, 40 * rows, 40_000 + 40 * rows)
        return _few_bytes(dict(kind=kind, rows=rows, table=rng.randint(64, 600), forks=forks, planes=rng.choice([2, 8, 32]),
                               pages=pages, page=page, kv_heads=kv_heads, dim=dim, dtype=dtype, fill=rng.uniform(0.1, 0.7)))
    if kind == "compact":
        rows = _log_int(rng, 4, 1000)
        return _few_bytes(dict(kind=kind, rows=rows, table=rng.randint(33, 300), forks=rng.randint(1, rows),
                               planes=rng.choice([2, 4, 8]), pages=_log_int(rng, 40 * rows, 65_536), page=page,
                               kv_heads=kv_heads, dim=dim, dtype=dtype, fill=rng.uniform(0.3, 0.95)))
    group = rng.choice([1, 2, 3, 4, 4, 8, 16])
    shape = rng.choice(["decode", "decode", "chunk", "chunk", "prefix"])
    c = dict(kind=kind, batch=1, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, heads=kv_heads * group, kv_heads=kv_heads, dim=dim,
             page=page, dtype=dtype, order=order, causal=shape != "prefix", holes=rng.random() < 0.2)
    if shape == "decode":
        c["batch"] = _log_int(rng, 1, 300)
        c["q_hi"] = rng.choice([1, 1, 1, 4])
        lo = _log_int(rng, 4, 60_000)
        c["kv_lo"], c["kv_hi"] = lo, _log_int(rng, lo, 2 * lo)
    elif shape == "chunk":
        c["batch"] = _log_int(rng, 1, 32)
        c["q_lo"] = rng.choice([1, _log_int(rng, 1, 2000)])
        c["q_hi"] = _log_int(rng, c["q_lo"], 4000)
        lo = rng.choice([c["q_hi"], _log_int(rng, c["q_hi"], 20_000)])
        c["kv_lo"], c["kv_hi"] = lo, _log_int(rng, lo, 2 * lo)
    else:
        c["q_lo"] = c["q_hi"] = _log_int(rng, 2, 500)
        c["kv_lo"] = c["kv_hi"] = _log_int(rng, 16, 40_000)
    while True:
        w = work(c)
        padded = c["batch"] * c["q_hi"] * c["heads"] * c["kv_hi"]
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and padded <= MOST_SCORES:
            return c
        if c["batch"] > 1:
            c["batch"] = c["batch"] * 2 // 3
        else:
            c["kv_hi"] = max(c["q_hi"], c["kv_hi"] * 2 // 3)
            c["kv_lo"] = min(c["kv_lo"], c["kv_hi"])
            if c["kv_hi"] == c["q_hi"]:
                c["q_hi"] = c["q_lo"] = max(1, c["q_hi"] * 2 // 3)


def _few_bytes(c):
    """A pool of at most 2.5 GB."""
    while c["planes"] * c["pages"] * 4 * c["page"] * c["kv_heads"] * c["dim"] > 2.5e9:
        if c["planes"] > 2:
            c["planes"] //= 2
        elif c["page"] > 8:
            c["page"] //= 2
        else:
            c["kv_heads"] = max(1, c["kv_heads"] // 2)
            c["dim"] = max(64, c["dim"] // 16 * 8)
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _lengths(c):
    """(new tokens, keys) per request: the same for every seed."""
    rng = random.Random(1000 * c["batch"] + c["kv_hi"])
    q = [rng.randint(c["q_lo"], c["q_hi"]) for _ in range(c["batch"])]
    return q, [max(n, rng.randint(c["kv_lo"], c["kv_hi"])) for n in q]


def _offsets(q):
    at = [0]
    for n in q:
        at.append(at[-1] + n)
    return at


def _pool(c, lead, pages, gen):
    """(whole pool, k view, v view): pages hold keys, then values; views [.., pages, page, kv_heads, dim]."""
    h, p = c["kv_heads"], c["page"]
    shape = (p, h) if c.get("order", "token") == "token" else (h, p)
    pool = torch.empty((*lead, pages, 2, *shape, c["dim"]), dtype=DTYPES[c["dtype"]], device="cuda")
    pool.normal_(generator=gen)
    k, v = pool.select(-4, 0), pool.select(-4, 1)
    if c.get("order", "token") == "head":
        k, v = k.transpose(-3, -2), v.transpose(-3, -2)
    return pool, k, v


def _prepare_sequences(c, gen):
    q, kv = _lengths(c)
    need = [-(-n // c["page"]) for n in kv]
    pages = sum(need) + sum(need) // 8 + 1
    pool, k, v = _pool(c, (), pages, gen)
    where = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at = torch.tensor(_offsets(need), device="cuda")
    i = torch.arange(max(need), device="cuda")
    table = torch.where(i < at.diff()[:, None], where[(at[:-1, None] + i).clamp(max=pages - 1)], -1)
    if c.get("holes"):  # pages that the cache has given up, some of them
        gone = torch.rand(table.shape, generator=gen, device="cuda") < 0.1
        table = torch.where(gone, -1, table)
    return dict(case=c, pool=pool, k=k, v=v, table=table.contiguous(), most_q=max(q), most_kv=max(kv), total=sum(q),
                q_offsets=torch.tensor(_offsets(q), dtype=torch.int32, device="cuda"),
                kv_lens=torch.tensor(kv, dtype=torch.int32, device="cuda"))


def _book_lengths(c):
    """(rows in use, tokens per row, pages per row): the same for every seed."""
    rows, width, p = c["rows"], c["table"], c["page"]
    live = rows - c["forks"] if c["kind"] == "fork" else rows  # the last rows are empty before a fork
    most = max(1, min(width - 4, int(c["fill"] * c["pages"]) // live))
    rng = random.Random(rows * 7 + width)
    lens = [rng.randint(max(1, p * most // 2), p * most) for _ in range(live)] + [0] * (rows - live)
    return live, lens, [-(-n // p) for n in lens]


def _prepare_book(c, gen):
    """A pool in use: `rows` table rows with pages of their own or a common prefix, free pages in between."""
    rows, width, pages, p = c["rows"], c["table"], c["pages"], c["page"]
    pool, _, _ = _pool(c, (c["planes"],), pages, gen)
    live, lens, need = _book_lengths(c)
    at = torch.tensor(_offsets(need), device="cuda")
    where = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    i = torch.arange(width, device="cuda")
    n = at.diff()[:, None]
    table = torch.where(i < n, where[(at[:-1, None] + i).clamp(max=pages - 1)], -1)
    # requests of a group share the first pages of the group's first row
    group = torch.arange(rows, device="cuda") // 8 * 8
    common = torch.minimum(n, n[group]) // 2
    table = torch.where(i < common, table[group], table)
    refs = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    refs.scatter_add_(0, torch.where(table >= 0, table, pages).long().reshape(-1), torch.ones_like(table).reshape(-1))
    book = torch.cat([table.reshape(-1), torch.tensor(lens, dtype=torch.int32, device="cuda"), refs[:pages]])
    work = torch.empty_like(book)
    t, l, r = work.split([rows * width, rows, pages])
    s = dict(case=c, pool=pool, book=book, work=work, table=t.view(rows, width), lens=l, refs=r)
    if c["kind"] == "fork":
        src = torch.randint(0, live, (c["forks"],), generator=gen, device="cuda")
        kept = (torch.rand(c["forks"], generator=gen, device="cuda") * (torch.tensor(lens, device="cuda")[src] + 1)).int()
        new = torch.randint(1, 3 * p, (c["forks"],), generator=gen, device="cuda", dtype=torch.int32)
        s.update(src=src.int(), dst=torch.arange(live, rows, device="cuda", dtype=torch.int32), keep=kept, new=new)
    else:
        s.update(gone=torch.randperm(rows, generator=gen, device="cuda")[: c["forks"]].int())
    return s


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if c["kind"] in ("fork", "compact"):
        return _prepare_book(c, gen)
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "merge":
        shape = (c["parts"], c["tokens"], c["heads"])
        lse = torch.randn(shape, generator=gen, device="cuda") * 2 + 7
        if c["empty"]:  # parts that hold no key for a row
            lse = torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.1, -math.inf, lse)
        outs = torch.randn((*shape, c["dim"]), generator=gen, device="cuda").to(dt)
        return dict(case=c, outs=outs, lses=lse)
    s = _prepare_sequences(c, gen)
    if c["kind"] == "write":
        shape = (2, s["total"], c["kv_heads"], c["dim"])
        new = torch.randn(shape, generator=gen, device="cuda").to(dt)
        s.update(k_new=new[0], v_new=new[1])
    else:
        s["q"] = (1.5 * torch.randn((s["total"], c["heads"], c["dim"]), generator=gen, device="cuda")).to(dt)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _where(s):
    """Request and position of every new token."""
    at = s["q_offsets"].long()
    t = torch.arange(s["total"], device="cuda")
    i = torch.searchsorted(at[1:].contiguous(), t, right=True)
    return i, t - at[i], s["kv_lens"].long()[i] - at.diff()[i] + t - at[i]


def _plain_attend(s):
    c = s["case"]
    b, h, hk, d, p = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    req, t, _ = _where(s)
    q = torch.zeros((b, s["most_q"], h, d), device="cuda")
    q[req, t] = s["q"].float()
    q = q.view(b, -1, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    table = s["table"].long()
    there = (table >= 0).repeat_interleave(p, 1)
    k = s["k"][table.clamp(min=0)].float().reshape(b, -1, hk, d).permute(0, 2, 3, 1)
    score = (q @ k).mul_(1 / math.sqrt(d)).view(b, hk, h // hk, s["most_q"], -1)
    del k
    j = torch.arange(there.shape[1], device="cuda")
    seen = there[:, None] & (j < s["kv_lens"][:, None, None])
    if c["causal"]:
        first = s["kv_lens"].long() - s["q_offsets"].long().diff()
        seen = seen & (j <= (first[:, None] + torch.arange(s["most_q"], device="cuda"))[:, :, None])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    e = score.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    v = s["v"][table.clamp(min=0)].float().reshape(b, -1, hk, d).permute(0, 2, 1, 3)
    o = (e.view(b, hk, -1, j.numel()) @ v).view(b, hk, h // hk, -1, d) / total.clamp(min=1e-30)
    out = o.permute(0, 3, 1, 2, 4).reshape(b, -1, h, d)[req, t].to(s["q"].dtype)
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(b, -1, h)[req, t]
    return dict(out=out, lse=lse)


def _plain_merge(s):
    lse, outs = s["lses"], s["outs"].float()
    top = lse.amax(0)
    top = torch.where(torch.isinf(top), 0.0, top)
    e = (lse - top).exp()
    total = e.sum(0)
    out = (outs * e[..., None]).sum(0) / total.clamp(min=1e-30)[..., None]
    return dict(out=out.to(s["outs"].dtype), lse=top + total.log())


def _plain_write(s):
    req, _, pos = _where(s)
    page = s["table"].long()[req, pos // s["case"]["page"]]
    s["k"][page, pos % s["case"]["page"]] = s["k_new"]
    s["v"][page, pos % s["case"]["page"]] = s["v_new"]
    return dict(k=s["k"], v=s["v"])


def _plain_fork(s):
    p, table, lens, refs = s["case"]["page"], s["table"], s["lens"], s["refs"]
    src, dst, keep = s["src"].long(), s["dst"].long(), s["keep"].long()
    i = torch.arange(table.shape[1], device="cuda")
    full, part = keep // p, keep % p > 0
    row = table[src]
    child = torch.where(i < full[:, None], row, -1)
    shared = child[child >= 0].long()
    free = (refs == 0).nonzero()[:, 0]
    fresh = free[(part.cumsum(0) - 1).clamp(min=0)]
    refs.scatter_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    refs[fresh[part]] = 1
    child[part, full[part]] = fresh[part].int()
    table[dst] = child
    lens[dst] = s["keep"]
    old = row[part, full[part]].long()
    s["pool"][:, fresh[part]] = s["pool"][:, old]
    # the forked rows grow
    more = lens[dst].long()
    have, want = -(-more // p), -(-(more + s["new"]) // p)
    grows = (i >= have[:, None]) & (i < want[:, None])
    free = (refs == 0).nonzero()[:, 0]
    got = free[: int((want - have).sum())]
    child = table[dst]
    child[grows] = got.int()
    table[dst] = child
    refs[got] = 1
    lens[dst] += s["new"]


def _plain_compact(s):
    table, lens, refs, gone = s["table"], s["lens"], s["refs"], s["gone"].long()
    row = table[gone]
    ids = row[row >= 0].long()
    refs.scatter_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
    table[gone] = -1
    lens[gone] = 0
    live = refs > 0
    n = int(live.sum())
    src = live[n:].nonzero()[:, 0] + n
    dst = (~live[:n]).nonzero()[:, 0]
    s["pool"][:, dst] = s["pool"][:, src]
    to = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    to[src] = dst.int()
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    refs[dst] = refs[src]
    refs[src] = 0


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if kind in ("fork", "compact"):
        s["work"].copy_(s["book"])  # the bookkeeping as it was; the pages that a pass writes are free again
    if own:
        from paper_2609_13692_gb300 import kv

        if kind == "attend":
            out, lse = kv.mpt_kv_attend(s["q"], s["k"], s["v"], s["table"], s["q_offsets"], s["kv_lens"],
                                        max_q_len=s["most_q"], causal=c["causal"])
            return dict(out=out, lse=lse)
        if kind == "merge":
            out, lse = kv.mpt_kv_merge(s["outs"], s["lses"])
            return dict(out=out, lse=lse)
        if kind == "write":
            kv.mpt_kv_write(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["q_offsets"], s["kv_lens"])
            return dict(k=s["k"], v=s["v"])
        book = (s["table"], s["lens"], s["refs"], c["page"])
        if kind == "fork":
            old, fresh, _ = kv.mpt_kv_fork(*book, s["src"], s["dst"], s["keep"])
            kv.mpt_kv_copy_pages(s["pool"], old, fresh)
            kv.mpt_kv_extend(*book, s["dst"], s["new"])
        else:
            kv.mpt_kv_free(*book, s["gone"])
            old, fresh, _ = kv.mpt_kv_compact(*book)
            kv.mpt_kv_copy_pages(s["pool"], old, fresh)
    elif kind == "attend":
        return _plain_attend(s)
    elif kind == "merge":
        return _plain_merge(s)
    elif kind == "write":
        return _plain_write(s)
    elif kind == "fork":
        _plain_fork(s)
    else:
        _plain_compact(s)
    return dict(table=s["table"], lens=s["lens"], refs=s["refs"], pool=s["pool"])


def work(case):
    """Inputs read once and outputs written once; products and sums over the pairs that are not masked."""
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "merge":
        rows = c["tokens"] * c["heads"]
        return {"bytes": (c["parts"] + 1) * rows * (c["dim"] * e + 4), "flops": 2 * c["parts"] * rows * c["dim"]}
    if c["kind"] in ("attend", "write"):
        q, kv = _lengths(c)
        tokens, table = sum(q), 4 * sum(-(-n // c["page"]) for n in kv)
        if c["kind"] == "write":
            return {"bytes": 4 * tokens * c["kv_heads"] * c["dim"] * e + 8 * c["batch"], "flops": 0}
        pairs = sum(n * t - n * (n - 1) // 2 if c["causal"] else n * t for n, t in zip(q, kv))
        rows = tokens * c["heads"]
        return {"bytes": 2 * sum(kv) * c["kv_heads"] * c["dim"] * e + rows * (2 * c["dim"] * e + 4) + table,
                "flops": 4 * c["dim"] * c["heads"] * pairs}
    page = 2 * c["page"] * c["kv_heads"] * c["dim"] * e * c["planes"]
    if c["kind"] == "fork":
        return {"bytes": 2 * c["forks"] * page * (c["page"] - 1) / c["page"] + 4 * c["pages"] + 8 * c["forks"] * c["table"],
                "flops": 0}
    # of the pages behind the live ones the live share moves; a group's common half is live while one of its rows is
    need, stay = _book_lengths(c)[2], 1 - c["forks"] / c["rows"]
    live = 0.0
    for first in range(0, len(need), 8):
        group = need[first:first + 8]
        common = [min(n, group[0]) // 2 for n in group[1:]]
        live += stay * (sum(group[1:]) - sum(common) + group[0] / 2) + (1 - (1 - stay) ** len(group)) * group[0] / 2
    live = live / c["pages"]
    return {"bytes": 2 * live * (1 - live) * c["pages"] * page + 12 * c["pages"] + 8 * c["rows"] * c["table"], "flops": 0}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, request by request and head by head
# ---------------------------------------------------------------------------

def exact(case, seed):
    c = dict(case)
    if c["kind"] not in ("attend", "merge"):
        return None  # pages and tables are moved, not computed
    s = prepare(case, seed)
    if c["kind"] == "merge":
        # weights of the parts by differences of their logarithms, part by part
        total = torch.full(s["lses"].shape[1:], -math.inf, dtype=torch.float64, device="cuda")
        for part in s["lses"]:
            total = torch.logaddexp(total, part.double())
        out = torch.zeros(s["outs"].shape[1:], dtype=torch.float64, device="cuda")
        for part, lse in zip(s["outs"], s["lses"]):
            out += torch.where(torch.isinf(lse), 0.0, (lse.double() - total).exp())[..., None] * part.double()
        return dict(out=out, lse=total)
    if work(c)["flops"] > 2e12:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    at, lens, group = s["q_offsets"].tolist(), s["kv_lens"].tolist(), c["heads"] // c["kv_heads"]
    for i in range(c["batch"]):
        j = torch.arange(lens[i], device="cuda")
        page = s["table"][i].long()[j // c["page"]]
        j, page = j[page >= 0], page[page >= 0]
        if not len(j):
            continue
        n = at[i + 1] - at[i]
        limit = lens[i] - n + torch.arange(n, device="cuda") if c["causal"] else torch.full((n,), lens[i], device="cuda")
        hidden = j[None] > limit[:, None]
        for g in range(c["kv_heads"]):
            k, v = s["k"][page, j % c["page"], g].double(), s["v"][page, j % c["page"], g].double()
            h = slice(g * group, (g + 1) * group)
            x = s["q"][at[i]:at[i + 1], h].double().transpose(0, 1) @ k.T / math.sqrt(c["dim"])
            x.masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(x, 2)
            lse[at[i]:at[i + 1], h] = z.T
            x = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[..., None])
            out[at[i]:at[i + 1], h] = (x @ v).transpose(0, 1)
    return dict(out=out, lse=lse)
