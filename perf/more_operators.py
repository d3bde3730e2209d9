"""Cases for measuring the operators that rotate keys on their way into the paged cache, and those of the
cache held in 4 bits: what a program that serves laid-out prompts does where positions are rotations and
where the cache, not the arithmetic, limits how many prompts it can hold.

New keys are rotated by their position, as the queries are, and written into pages, in 16 bits or as codes
of 4 bits; new tokens attend over the codes; and what was written is read back where a request is handed to
a cache of 16 bits.  Lengths go with the repository's workloads: groups of 12 to 28 requests of 5 to 20
passages of about 150 tokens, and long streams.  All inputs are synthetic, drawn from the seed.

A page of the 4-bit cache holds, for each KV head, tiles of 8 tokens.  With n = ceil(dim / 32) groups of 32
elements, a tile is: codes of keys [8][16 n], of their groups the scale and offset [8][n][2], codes of values
[4 pairs of tokens][8 n pieces of 4 elements][2 tokens][2], scales and offsets of values [4][n][2][2 tokens].
Four codes are 16 bits, the first the lowest, rotated left by six bits.  A scale byte is the upper part of a
positive half-precision number a (5 bits of exponent, 3 of mantissa), an offset byte z + 128; code c stands
for (c + z) a / 16.
"""

import math
import random

import torch

own = False  # False: the operators in elementary torch operations, in 32 bits; True: the framework's kernels

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}

LISTED = [
    # One new token for each of the 28 requests of the benchmark's group: queries and keys rotated, keys and
    # values appended; nothing but latency.
    dict(name="rotate_m28", kind="rotate", batch=28, q_lo=1, q_hi=1, kv_lo=2000, kv_hi=6000, heads=32, kv_heads=8, dim=128,
         rot=128, adjacent=False, places=False, page=16, dtype="bf16", holes=False),
    # The new tokens of a prefill step of 28 requests.
    dict(name="rotate_prefill", kind="rotate", batch=28, q_lo=300, q_hi=2100, kv_lo=2200, kv_hi=4000, heads=32, kv_heads=8,
         dim=128, rot=128, adjacent=False, places=False, page=16, dtype="bf16", holes=False),
    # Ragged chunks of a model that turns adjacent elements of half of each head, at positions of the
    # caller's choice (passages cached at places of their own); a tenth of the pages absent.
    dict(name="rotate_ragged", kind="rotate", batch=13, q_lo=1, q_hi=700, kv_lo=700, kv_hi=6000, heads=24, kv_heads=8, dim=96,
         rot=48, adjacent=True, places=True, page=32, dtype="f16", holes=True),
    # The same steps where the cache holds 4-bit codes: next tokens of many requests, appended and read back.
    dict(name="codes_m200", kind="codes", batch=200, q_lo=1, q_hi=1, kv_lo=200, kv_hi=400, heads=32, kv_heads=8, dim=128,
         rot=128, adjacent=False, places=False, page=16, dtype="bf16", holes=False),
    # A prefill step into 4 bits, and its values back.
    dict(name="codes_prefill", kind="codes", batch=28, q_lo=300, q_hi=2100, kv_lo=2200, kv_hi=4000, heads=32, kv_heads=8,
         dim=128, rot=128, adjacent=False, places=False, page=16, dtype="bf16", holes=False),
    # Heads that are no whole number of groups, no rotation, the smallest pages, some of them absent.
    dict(name="codes_odd", kind="codes", batch=19, q_lo=1, q_hi=333, kv_lo=333, kv_hi=1999, heads=6, kv_heads=6, dim=80,
         rot=0, adjacent=False, places=False, page=8, dtype="f16", holes=True),
    # One request's next token over a prompt of a few passages: nothing but latency.
    dict(name="decode_one", kind="attend", batch=1, q_lo=1, q_hi=1, kv_lo=777, kv_hi=777, heads=32, kv_heads=8, dim=128,
         page=16, dtype="bf16", causal=True, holes=False),
    # The benchmark's group of 28 requests, each at its next token over its prompt of 20 passages.
    dict(name="decode_m28", kind="attend", batch=28, q_lo=1, q_hi=1, kv_lo=2000, kv_hi=6000, heads=32, kv_heads=8, dim=128,
         page=16, dtype="bf16", causal=True, holes=False),
    # Few requests over very long contexts (a million-passage workload's deep retrieval), 64-token pages.
    dict(name="decode_long", kind="attend", batch=3, q_lo=1, q_hi=1, kv_lo=100_001, kv_hi=131_072, heads=64, kv_heads=8,
         dim=128, page=64, dtype="f16", causal=True, holes=False),
    # Many requests at up to four tokens each (drafts to be checked), small heads in pairs.
    dict(name="decode_drafts", kind="attend", batch=150, q_lo=1, q_hi=4, kv_lo=300, kv_hi=5000, heads=32, kv_heads=16, dim=64,
         page=32, dtype="bf16", causal=True, holes=False),
    # 28 requests in one step of a continuous batch: some at one token, others with up to 700 new ones; odd head size.
    dict(name="chunk_ragged", kind="attend", batch=28, q_lo=1, q_hi=700, kv_lo=700, kv_hi=6000, heads=24, kv_heads=8, dim=96,
         page=32, dtype="f16", causal=True, holes=True),
    # A long prompt's chunk: 4,096 new tokens over 16,384 cached ones.
    dict(name="chunk_long", kind="attend", batch=1, q_lo=4096, q_hi=4096, kv_lo=20_480, kv_hi=20_480, heads=32, kv_heads=8,
         dim=128, page=16, dtype="bf16", causal=True, holes=False),
]


def listed():
    return [dict(c) for c in LISTED]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST_FLOPS = 1.0e12   # of a drawn attention (chunk_long: 1.2e12)
MOST_BYTES = 3.5e8    # (decode_long: 4e8; rotate_prefill 8e8)
MOST_SCORES = 4.0e9   # entries of the plain form's score matrix, padding among them
MOST_KEYS = 4.0e8     # elements of keys that the plain form widens, padding among them


def draw(rng):
    kind = rng.choice(["rotate", "codes", "attend", "attend"])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    group = rng.choice([1, 2, 3, 4, 4, 8, 16])
    dim = rng.choice([64, 128, 128, 128, 96, 80, 40, 192, 256])
    c = dict(kind=kind, batch=1, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, heads=kv_heads * group, kv_heads=kv_heads, dim=dim,
             page=rng.choice([8, 16, 16, 32, 64, 128, 256]), dtype=rng.choice(["bf16", "f16"]), holes=rng.random() < 0.2)
    if kind != "attend":
        adjacent = rng.random() < 0.4
        unit = 8 if adjacent else 16
        turned = rng.choice([dim, dim, dim // 2, unit]) // unit * unit
        c.update(adjacent=adjacent, rot=0 if kind == "codes" and rng.random() < 0.2 else max(unit, turned),
                 places=rng.random() < 0.3)
        lo = _log_int(rng, 1, 1000)
        c.update(batch=_log_int(rng, 1, 256), q_lo=lo, q_hi=_log_int(rng, lo, 2 * lo + 1), kv_lo=2 * lo + 1,
                 kv_hi=_log_int(rng, 2 * lo + 1, 6000))
        while work(c)["bytes"] > MOST_BYTES:
            c["batch"] = c["batch"] * 2 // 3
        return c
    shape = rng.choice(["decode", "decode", "chunk", "chunk", "prefix"])
    c["causal"] = shape != "prefix"
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
        wide = c["batch"] * c["kv_heads"] * c["dim"] * c["kv_hi"]
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and padded <= MOST_SCORES and wide <= MOST_KEYS:
            return c
        if c["batch"] > 1:
            c["batch"] = c["batch"] * 2 // 3
        else:
            c["kv_hi"] = max(c["q_hi"], c["kv_hi"] * 2 // 3)
            c["kv_lo"] = min(c["kv_lo"], c["kv_hi"])
            if c["kv_hi"] == c["q_hi"]:
                c["q_hi"] = c["q_lo"] = max(1, c["q_hi"] * 2 // 3)


# ---------------------------------------------------------------------------
# The 4-bit cache
# ---------------------------------------------------------------------------

def _groups(dim):
    return -(-dim // 32)


def page_bytes(page, dim):
    return page // 8 * 288 * _groups(dim)


def _parts(pages, dim):
    """Views of pages [.., bytes]: codes of keys [.., tiles, 8, 16 n], their scales and offsets [.., 8, n, 2], codes
    of values [.., tiles, 4, 8 n, 2 tokens, 2], their scales and offsets [.., 4, n, 2, 2 tokens]."""
    n = _groups(dim)
    t = pages.unflatten(-1, (-1, 288 * n))
    return (t[..., :128 * n].unflatten(-1, (8, 16 * n)), t[..., 128 * n:144 * n].unflatten(-1, (8, n, 2)),
            t[..., 144 * n:272 * n].unflatten(-1, (4, 8 * n, 2, 2)), t[..., 272 * n:].unflatten(-1, (4, n, 2, 2)))


def _quantise(x):
    """x: [.., dim] of 32 bits; (codes [.., 8 n pieces, 2 bytes], scale and offset bytes [.., n, 2])."""
    n = _groups(x.shape[-1])
    x = torch.nan_to_num(x, nan=0.0).clamp(-3360.0, 3360.0)
    short = 32 * n - x.shape[-1]
    if short:  # the last group's missing elements are like its first
        x = torch.cat([x, x[..., -(32 - short)].unsqueeze(-1).expand(*x.shape[:-1], short)], -1)
    x = x.unflatten(-1, (n, 32))
    lo, hi = x.amin(-1), x.amax(-1)
    # divided by tensors: by a number, torch multiplies with its inverse on a GPU, and many steps stand on a border
    step = torch.maximum((hi - lo) / torch.full_like(lo, 15.0), torch.maximum(hi, -lo) / torch.full_like(lo, 120.0))
    step = step.clamp(min=2.0 ** -18)
    step = ((step.view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32)  # up to 3 bits of mantissa
    z = (lo / step).round()
    c = ((x / step[..., None]).round() - z[..., None]).clamp(0, 15)
    scale = ((16 * step).view(torch.int32) >> 20) - ((127 - 15) << 3)
    c = c.int().unflatten(-1, (8, 4))
    half = c[..., 0] | c[..., 1] << 4 | c[..., 2] << 8 | c[..., 3] << 12
    half = (half << 6 | half >> 10) & 0xFFFF
    codes = torch.stack([half & 255, half >> 8], -1).to(torch.uint8).flatten(-3, -2)
    return codes, torch.stack([scale, z.int() + 128], -1).to(torch.uint8)


def _values(codes, marks, dim):
    """The 32-bit values of codes [.., 8 n, 2] with scale and offset bytes [.., n, 2]; [.., dim]."""
    n = _groups(dim)
    half = codes[..., 0].int() | codes[..., 1].int() << 8
    half = (half >> 6 | half << 10) & 0xFFFF
    c = torch.stack([half & 15, half >> 4 & 15, half >> 8 & 15, half >> 12], -1).float()
    a = (marks[..., 0].int() + ((127 - 15) << 3) << 20).view(torch.float32) / 16
    z = marks[..., 1].float() - 128
    c = c.unflatten(-2, (n, 8)).flatten(-2)
    return ((c + z[..., None]) * a[..., None]).flatten(-2)[..., :dim]


def _put(pages, dim, page, at, k, v):
    """Keys and values [tokens, kv_heads, dim] (32 bits) into place `at` of their pages."""
    kc, km, vc, vm = _parts(pages, dim)
    t, s = at // 8, at % 8
    codes, marks = _quantise(k)
    kc[page, :, t, s] = codes.flatten(-2)
    km[page, :, t, s] = marks
    codes, marks = _quantise(v)
    vc[page, :, t, s // 2, :, s % 2] = codes
    vm[page, :, t, s // 2, :, :, s % 2] = marks


def _get(pages, dim, page, at):
    kc, km, vc, vm = _parts(pages, dim)
    t, s = at // 8, at % 8
    return (_values(kc[page, :, t, s].unflatten(-1, (-1, 2)), km[page, :, t, s], dim),
            _values(vc[page, :, t, s // 2, :, s % 2], vm[page, :, t, s // 2, :, :, s % 2], dim))


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


def _turns(rows, rot):
    """Cosines, then sines, of every position's angles; the angles in 64 bits."""
    rate = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * rate
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, h, p, dim = DTYPES[c["dtype"]], c["kv_heads"], c["page"], c["dim"]
    q, kv = _lengths(c)
    need = [-(-n // p) for n in kv]
    pages = sum(need) + sum(need) // 8 + 1
    where = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at = torch.tensor(_offsets(need), device="cuda")
    i = torch.arange(max(need), device="cuda")
    table = torch.where(i < at.diff()[:, None], where[(at[:-1, None] + i).clamp(max=pages - 1)], -1)
    if c["holes"]:  # pages that the cache has given up, some of them
        table = torch.where(torch.rand(table.shape, generator=gen, device="cuda") < 0.1, -1, table)
    total = sum(q)
    s = dict(case=c, table=table.contiguous(), most_q=max(q), most_kv=max(kv), total=total,
             q_offsets=torch.tensor(_offsets(q), dtype=torch.int32, device="cuda"),
             kv_lens=torch.tensor(kv, dtype=torch.int32, device="cuda"))
    s["q"] = (1.5 * torch.randn((total, c["heads"], dim), generator=gen, device="cuda")).to(dt)
    if c["kind"] == "rotate":
        pool = torch.empty((pages, 2, p, h, dim), dtype=dt, device="cuda")
        pool.normal_(generator=gen)
        s.update(pool=pool, k=pool[:, 0], v=pool[:, 1])
    else:
        s["pages"] = torch.zeros((pages, h, page_bytes(p, dim)), dtype=torch.uint8, device="cuda")
        some = max(1, 30_000_000 // (p * h * dim))
        for first in range(0, pages, some):
            n = min(some, pages - first)
            x = torch.randn((2, n * p, h, dim), generator=gen, device="cuda")
            j = torch.arange(n * p, device="cuda")
            _put(s["pages"], dim, first + j // p, j % p, x[0], x[1])
    if c["kind"] != "attend":
        new = torch.randn((2, total, h, dim), generator=gen, device="cuda").to(dt)
        s.update(k_new=new[0], v_new=new[1], places=None, turns=None)
        if c["rot"]:
            s["turns"] = _turns(max(kv), c["rot"])
            if c["places"]:
                s["places"] = torch.randint(0, max(kv), (total,), generator=gen, device="cuda", dtype=torch.int32)
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


def _turned(x, turn, c):
    """x [tokens, heads, dim] in 32 bits, turned by the rows [tokens, rot] of cosines and sines."""
    x, r = x.float(), c["rot"]
    if not r:
        return x
    cos, sin = turn[:, None, :r // 2], turn[:, None, r // 2:]
    if c["adjacent"]:
        one, two = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([one * cos - two * sin, two * cos + one * sin], -1).flatten(-2)
    else:
        one, two = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([one * cos - two * sin, two * cos + one * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_append(s):
    c = s["case"]
    dt, p = s["q"].dtype, c["page"]
    req, _, pos = _where(s)
    turn = None if s["turns"] is None else s["turns"][pos if s["places"] is None else s["places"].long()]
    k, v = _turned(s["k_new"], turn, c), s["v_new"]
    out = dict(q=_turned(s["q"], turn, c).to(dt)) if c["rot"] else {}
    page = s["table"].long()[req, pos // p]
    on = page >= 0
    if c["kind"] == "rotate":
        s["k"][page[on], pos[on] % p] = k[on].to(dt)
        s["v"][page[on], pos[on] % p] = v[on]
        return dict(out, k=s["k"], v=s["v"])
    _put(s["pages"], c["dim"], page[on], pos[on] % p, k[on], v[on].float())
    got = _get(s["pages"], c["dim"], page.clamp(min=0), pos % p)
    k, v = (torch.where(on[:, None, None], x, 0.0).to(dt) for x in got)
    return dict(out, k=k, v=v)


def _plain_attend(s):
    c = s["case"]
    b, h, hk, d, p = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    req, t, _ = _where(s)
    q = torch.zeros((b, s["most_q"], h, d), device="cuda")
    q[req, t] = s["q"].float()
    q = q.view(b, -1, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    table = s["table"].long()
    there = (table >= 0).repeat_interleave(p, 1)
    kc, km, vc, vm = _parts(s["pages"][table.clamp(min=0)].transpose(1, 2), d)  # [batch, kv_heads, pages of a row, tiles, ..]
    k = _values(kc.unflatten(-1, (-1, 2)), km, d).reshape(b, hk, -1, d)
    score = (q @ k.transpose(2, 3)).mul_(1 / math.sqrt(d)).view(b, hk, h // hk, s["most_q"], -1)
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
    v = _values(vc.transpose(-3, -2), vm.movedim(-1, -3), d).reshape(b, hk, -1, d)
    o = (e.view(b, hk, -1, j.numel()) @ v).view(b, hk, h // hk, -1, d) / total.clamp(min=1e-30)
    out = o.permute(0, 3, 1, 2, 4).reshape(b, -1, h, d)[req, t].to(s["q"].dtype)
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(b, -1, h)[req, t]
    return dict(out=out, lse=lse)


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2609_13692_gb300 import kv

        where = (s["table"], s["q_offsets"], s["kv_lens"])
        if c["kind"] == "attend":
            out, lse = kv.mpt_kv4_attend(s["q"], s["pages"], *where, max_q_len=s["most_q"], causal=c["causal"])
            return dict(out=out, lse=lse)
        if c["kind"] == "rotate":
            q = kv.mpt_kv_write_rotated(s["k_new"], s["v_new"], s["turns"], s["k"], s["v"], *where, q=s["q"],
                                        positions=s["places"], adjacent=c["adjacent"])
            return dict(q=q, k=s["k"], v=s["v"])
        q = kv.mpt_kv4_write(s["k_new"], s["v_new"], s["pages"], *where, rotation=s["turns"], q=s["q"] if c["rot"] else None,
                             positions=s["places"], adjacent=c["adjacent"])
        k, v = kv.mpt_kv4_read(s["pages"], *where, s["total"], c["dim"], dtype=s["q"].dtype)
        return dict(q=q, k=k, v=v) if c["rot"] else dict(k=k, v=v)
    return _plain_attend(s) if c["kind"] == "attend" else _plain_append(s)


def work(case):
    """Inputs read once and outputs written once; products and sums over the pairs that are not masked."""
    c = case
    q, kv = _lengths(c)
    tokens, table, n = sum(q), 4 * sum(-(-x // c["page"]) for x in kv), _groups(c["dim"])
    if c["kind"] != "attend":
        new = 4 * tokens * c["kv_heads"] * c["dim"]  # keys and values, in 16 bits
        queries = 4 * tokens * c["heads"] * c["dim"] + 4 * tokens * c["rot"] if c["rot"] else 0
        # the 16-bit cache is what is written; of codes both they and the values that are read back
        codes = 36 * n * tokens * c["kv_heads"] if c["kind"] == "codes" else 0
        return {"bytes": 2 * new + queries + codes + 8 * c["batch"], "flops": 0}
    pairs = sum(m * t - m * (m - 1) // 2 if c["causal"] else m * t for m, t in zip(q, kv))
    rows = tokens * c["heads"]
    return {"bytes": 36 * n * sum(kv) * c["kv_heads"] + rows * (4 * c["dim"] + 4) + table,
            "flops": 4 * c["dim"] * c["heads"] * pairs}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_turn(x, turn, c):
    """Rotation as the product of complex numbers."""
    x, r = x.double(), c["rot"]
    if not r:
        return x
    w = torch.complex(turn[:, :r // 2].double(), turn[:, r // 2:].double())[:, None]
    if c["adjacent"]:
        y = torch.view_as_real(torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * w).flatten(-2)
    else:
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * w
        y = torch.cat([z.real, z.imag], -1)
    return torch.cat([y, x[..., r:]], -1)


def _exact_round(x):
    """The nearest value that the 4-bit cache can hold for each element of x [.., dim], group by group."""
    done = []
    for first in range(0, x.shape[-1], 32):
        g = x[..., first:first + 32]
        lo, hi = g.min(-1, keepdim=True)[0], g.max(-1, keepdim=True)[0]
        step = torch.maximum((hi - lo) / 15, torch.maximum(hi.abs(), lo.abs()) / 120).clamp(min=2.0 ** -18)
        e = torch.floor(torch.log2(step)) - 3
        step = torch.ceil(step * torch.exp2(-e)) * torch.exp2(e)
        z = torch.round(lo / step)
        done.append((z + torch.minimum(torch.round(g / step) - z, torch.full_like(g, 15.0))) * step)
    return torch.cat(done, -1)


def _exact_tile(raw, n, dim, value):
    """The 64-bit values [tiles, 8, dim] of keys or values of tiles [tiles, 288 n]."""
    raw = raw.long()
    e = torch.arange(32 * n, device="cuda")
    tok = torch.arange(8, device="cuda")[:, None]
    g = e // 32
    if value:
        at = 144 * n + tok // 2 * 32 * n + e // 4 * 4 + tok % 2 * 2
        mark = 272 * n + tok // 2 * 4 * n + g * 4 + tok % 2
        scale, offset = raw[:, mark], raw[:, mark + 2]
    else:
        at = tok * 16 * n + e // 4 * 2
        mark = 128 * n + tok * 2 * n + g * 2
        scale, offset = raw[:, mark], raw[:, mark + 1]
    half = raw[:, at] + 256 * raw[:, at + 1]
    code = (half * 65537 >> (6 + 4 * (e % 4))) & 15  # of the 16 bits twice over
    a = torch.exp2((scale // 8).double() - 15) * (1 + (scale % 8).double() / 8)
    return ((code + offset - 128).double() * a / 16)[..., :dim]


def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["kind"] != "attend":
        at, lens = s["q_offsets"].tolist(), s["kv_lens"].tolist()
        pos = torch.cat([torch.arange(n - (b - a), n, device="cuda") for a, b, n in zip(at, at[1:], lens)])
        req = torch.cat([torch.full((b - a,), i, device="cuda") for i, (a, b) in enumerate(zip(at, at[1:]))])
        turn = s["turns"][s["places"].long() if s["places"] is not None else pos] if c["rot"] else None
        page = s["table"][req, pos // c["page"]].long()
        k, v = _exact_turn(s["k_new"], turn, c), s["v_new"].double()
        out = dict(q=_exact_turn(s["q"], turn, c)) if c["rot"] else {}
        if c["kind"] == "codes":
            gone = (page < 0)[:, None, None]
            return dict(out, k=_exact_round(k).masked_fill(gone, 0.0), v=_exact_round(v).masked_fill(gone, 0.0))
        held = torch.nonzero(page >= 0)[:, 0]
        place = page[held] * c["page"] + pos[held] % c["page"]
        flat = (s["k"].double().flatten(0, 1), s["v"].double().flatten(0, 1))
        for whole, x in zip(flat, (k, v)):
            whole.index_copy_(0, place, x[held])
        return dict(out, k=flat[0].view(s["k"].shape), v=flat[1].view(s["v"].shape))
    if work(c)["flops"] > 2e12:
        return None
    n = _groups(c["dim"])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    at, lens, group = s["q_offsets"].tolist(), s["kv_lens"].tolist(), c["heads"] // c["kv_heads"]
    for i in range(c["batch"]):
        row = s["table"][i].long()
        held = torch.nonzero(row >= 0)[:, 0]
        j = (held[:, None] * c["page"] + torch.arange(c["page"], device="cuda")).flatten()
        live = torch.nonzero(j < lens[i])[:, 0]
        if not len(live):
            continue
        m = at[i + 1] - at[i]
        limit = lens[i] - m + torch.arange(m, device="cuda") if c["causal"] else torch.full((m,), lens[i], device="cuda")
        hidden = j[live][None] > limit[:, None]
        for g in range(c["kv_heads"]):
            raw = s["pages"][row[held], g].reshape(-1, 288 * n)
            k = _exact_tile(raw, n, c["dim"], False).flatten(0, 1)[live]
            v = _exact_tile(raw, n, c["dim"], True).flatten(0, 1)[live]
            h = slice(g * group, (g + 1) * group)
            x = s["q"][at[i]:at[i + 1], h].double().transpose(0, 1) @ k.T / math.sqrt(c["dim"])
            x.masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(x, 2)
            lse[at[i]:at[i + 1], h] = z.T
            x = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[..., None])
            out[at[i]:at[i + 1], h] = (x @ v).transpose(0, 1)
    return dict(out=out, lse=lse)
