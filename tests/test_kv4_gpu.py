"""The turned writes and the cache in 4 bits against their models: bits of pages, values read back, and
attention in 64 bits over them."""

import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import kv4_model as K
from tests import kv_model as M

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def kv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    B.build()
    from paper_2609_13692_gb300 import kv as K

    return K


def layout(seed, q_lens, kv_lens, page, holes=0.0, spare=3, pad=0):
    """(table, q_offsets, kv_lens, n_pages): pages in random order, some of them absent."""
    rng = random.Random(seed)
    need = [-(-n // page) for n in kv_lens]
    n_pages = sum(need) + spare
    ids = list(range(n_pages))
    rng.shuffle(ids)
    table = torch.full((len(kv_lens), max([1, *need]) + 1 + pad), n_pages + 5, dtype=torch.int32)
    for i, n in enumerate(need):
        for t in range(n):
            p = ids.pop()
            table[i, t] = rng.choice([-1, n_pages, -2 ** 31, 2 ** 31 - 1]) if rng.random() < holes else p
    at = np.concatenate([[0], np.cumsum(q_lens)]) if q_lens else np.zeros(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    return table.cuda()[:, :table.shape[1] - pad], torch.tensor(at.astype(np.int32), **i32), torch.tensor(kv_lens, **i32), n_pages


def places(table, at, lens, page, tokens, n_pages):
    """Per token: request (-1: none), position, page id (-1: none)."""
    table, at, lens = table.cpu().tolist(), at.tolist(), lens.tolist()
    found = [(-1, 0, -1)] * tokens
    for i, n in enumerate(lens):
        for t in range(at[i], min(at[i + 1], tokens)):
            pos = n - (at[i + 1] - at[i]) + t - at[i]
            id = table[i][pos // page] if 0 <= pos < page * len(table[i]) else -1
            found[t] = (i, pos, id if 0 <= id < n_pages else -1)
    return found


def hard(gen, shape, dtype):
    """Ordinary values, groups of equal ones, of one sign, far from 0, tiny, huge, NaN and infinities."""
    x = torch.randn(shape, generator=gen, device="cuda")
    pick = torch.randint(0, 12, shape[:2], generator=gen, device="cuda")[..., None]
    x = torch.where(pick == 1, 0.25 * x.round(), x)
    x = torch.where(pick == 2, 3.0, x)
    x = torch.where(pick == 3, x.abs() + 50, x)
    x = torch.where(pick == 4, -x.abs(), x)
    x = torch.where(pick == 5, x * 1e-6, x)
    x = torch.where(pick == 6, x * 3000, x)
    x = torch.where(pick == 7, torch.zeros_like(x), x)
    x = x.to(dtype)
    if shape[0] and shape[2] > 1:
        flat = x.view(-1)
        at = torch.randint(0, flat.numel(), (5,), generator=gen, device="cuda")
        flat[at] = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0], device="cuda").to(dtype)
    return x


def strided(x, order):
    """The same values with gaps between tokens and heads, or heads before tokens."""
    if order == "gaps":
        wide = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + 8), 7.0, dtype=x.dtype, device=x.device)
        wide[:, :-1, :x.shape[2]] = x
        return wide[:, :-1, :x.shape[2]]
    if order == "head":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    return x


WRITES = [  # q_lens, kv_lens, heads, kv_heads, dim, page, rot, adjacent, places, order
    ([1, 1, 1], [1, 17, 300], 4, 2, 128, 16, 128, False, False, "plain"),
    ([5, 0, 40, 3], [5, 9, 60, 1], 6, 3, 96, 8, 48, True, True, "gaps"),
    ([33], [40], 2, 1, 256, 256, 256, False, False, "head"),
    ([7, 9], [7, 900], 5, 5, 8, 32, 8, True, False, "gaps"),
    ([20, 2], [64, 2], 9, 3, 80, 16, 16, False, True, "plain"),
    ([3, 1, 2], [9, 1, 2], 3, 1, 40, 64, 32, False, False, "head"),
    ([4], [130], 7, 7, 200, 128, 200, True, False, "plain"),
]


def write_case(seed, case, dtype, holes):
    q_lens, kv_lens, heads, kv_heads, dim, page, rot, adjacent, own_places, order = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table, at, lens, n_pages = layout(seed, q_lens, kv_lens, page, holes)
    tokens = sum(q_lens) + 2  # two of no request
    x = [strided(hard(gen, (tokens, h, dim), dtype), order) for h in (heads, kv_heads, kv_heads)]
    rows = max(kv_lens) - (1 if max(kv_lens) > 20 else 0)  # the last position may have no row
    turns = torch.zeros((rows, rot + 4), device="cuda")[:, :rot]
    turns.copy_(torch.from_numpy(K.angles(rows, rot)))
    pos = torch.randint(-1, rows + 1, (tokens,), generator=gen, device="cuda", dtype=torch.int32) if own_places else None
    where = places(table, at, lens, page, tokens, n_pages)
    at_rows = np.array([p for _, p, _ in where]) if pos is None else pos.cpu().numpy()
    return dict(x=x, table=table, at=at, lens=lens, n_pages=n_pages, turns=turns, pos=pos, where=where, rows=at_rows, page=page,
                dim=dim, rot=rot, adjacent=adjacent, kv_heads=kv_heads)


def same(a, b):
    """Equal bits, or both NaN."""
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def expected_q(c, got):
    """The turned queries, and what stood in the output for tokens of no request."""
    q = c["x"][0]
    want = torch.from_numpy(K.turned(q.float().cpu().numpy(), c["turns"].cpu().numpy(), c["rows"], c["rot"], c["adjacent"])).to(q.dtype)
    mine = torch.tensor([r >= 0 for r, _, _ in c["where"]])
    assert same(got.cpu()[mine], want[mine])
    return mine


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("case", WRITES, ids=range(len(WRITES)))
def test_rotated_writes(kv, case, dtype):
    for holes in (0.0, 0.3):
        c = write_case(1, case, dtype, holes)
        q, k_new, v_new = c["x"]
        pool = torch.full((c["n_pages"], 2, c["page"], c["kv_heads"], c["dim"]), 9.0, dtype=dtype, device="cuda")
        want = pool.cpu().clone()
        out = torch.full(q.shape, -5.0, dtype=dtype, device="cuda")
        back = kv.mpt_kv_write_rotated(k_new, v_new, c["turns"], pool[:, 0], pool[:, 1], c["table"], c["at"], c["lens"], q=q,
                                       positions=c["pos"], adjacent=c["adjacent"], q_out=out)
        kv.mpt_kv_check()
        assert back is out
        mine = expected_q(c, out)
        assert bool((out.cpu()[~mine] == -5.0).all())
        k = torch.from_numpy(K.turned(k_new.float().cpu().numpy(), c["turns"].cpu().numpy(), c["rows"], c["rot"], c["adjacent"])).to(dtype)
        for t, (_, pos, id) in enumerate(c["where"]):
            if id >= 0 and 0 <= c["rows"][t] < len(c["turns"]):
                want[id, 0, pos % c["page"]], want[id, 1, pos % c["page"]] = k[t], v_new[t].cpu()
        assert same(pool.cpu(), want)


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("case", WRITES, ids=range(len(WRITES)))
def test_codes(kv, case, dtype, turned):
    """Every byte of the pages, and what is read back in three types."""
    c = write_case(2, case, dtype, 0.2)
    q, k_new, v_new = c["x"]
    size = kv.mpt_kv4_page_bytes(c["page"], c["dim"])
    whole = torch.randint(0, 256, (c["n_pages"], c["kv_heads"], size + 32), dtype=torch.uint8, device="cuda")  # heads with gaps
    pages = whole[:, :, :size]
    want = pages.cpu().numpy().copy()
    more = dict(rotation=c["turns"], q=q, positions=c["pos"], adjacent=c["adjacent"]) if turned else {}
    out = kv.mpt_kv4_write(k_new, v_new, pages, c["table"], c["at"], c["lens"], **more)
    kv.mpt_kv_check()
    k = k_new.float().cpu().numpy()
    if turned:
        expected_q(c, out)
        with np.errstate(invalid="ignore"):
            k = K.turned(k, c["turns"].cpu().numpy(), c["rows"], c["rot"], c["adjacent"])
    else:
        assert out is None
    v = v_new.float().cpu().numpy()
    held = []
    for t, (_, pos, id) in enumerate(c["where"]):
        here = id >= 0 and (not turned or 0 <= c["rows"][t] < len(c["turns"]))
        held.append(here)
        for h in range(c["kv_heads"] if here else 0):
            K.put(want, c["dim"], id, pos % c["page"], h, k[t, h], v[t, h])
    assert np.array_equal(pages.cpu().numpy(), want)
    vals = K.values(torch.from_numpy(want), c["dim"])
    for dt in (BF16, F16, torch.float32):
        outs = [torch.full(k_new.shape, -3.0, dtype=dt, device="cuda") for _ in range(2)]
        kv.mpt_kv4_read(pages, c["table"], c["at"], c["lens"], len(k_new), c["dim"], dtype=dt, k_out=outs[0], v_out=outs[1])
        kv.mpt_kv_check()
        for got, x in zip(outs, vals):
            for t, (r, pos, id) in enumerate(c["where"]):
                w = torch.full(x.shape[2:], -3.0) if r < 0 else x[id, pos % c["page"]] if id >= 0 else torch.zeros(x.shape[2:])
                assert torch.equal(got[t].cpu(), w.to(dt)), t


def test_turned_in_place_and_in_part(kv):
    """Queries turned where they stand, as views of one packed tensor; the same tokens in two calls."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens, heads, kv_heads, dim = 50, 8, 2, 128
    table, at, lens, n_pages = layout(3, [20, 30], [90, 30], 16)
    turns = torch.from_numpy(K.angles(100, dim)).cuda()
    packed = torch.randn((tokens, heads + 2 * kv_heads, dim), generator=gen, device="cuda").to(BF16)
    pool = torch.zeros((n_pages, 2, 16, kv_heads, dim), dtype=BF16, device="cuda")
    views = lambda x: (x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:])  # noqa: E731
    q, k, v = views(packed.clone())
    want = kv.mpt_kv_write_rotated(k, v, turns, pool[:, 0], pool[:, 1], table, at, lens, q=q)
    same_pool = torch.zeros_like(pool)
    mine = packed.clone()
    q, k, v = views(mine)
    assert kv.mpt_kv_write_rotated(k, v, turns, same_pool[:, 0], same_pool[:, 1], table, at, lens, q=q, q_out=q) is q
    assert torch.equal(q, want) and torch.equal(pool, same_pool)
    assert torch.equal(mine[:, heads:], packed[:, heads:])
    assert kv.mpt_kv_write_rotated(k, v, turns, same_pool[:, 0], same_pool[:, 1], table, at, lens) is None


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def make(seed, q_lens, kv_lens, heads, kv_heads, dim, page, dtype, holes=0.0, spread=1.0):
    """A cache of codes of normal values, any bytes where nothing is stored."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table, at, lens, n_pages = layout(seed, q_lens, kv_lens, page, holes, pad=seed % 2)
    n = K.groups(dim)
    pages = torch.randint(0, 256, (n_pages, kv_heads, page // 8 * 288 * n), generator=gen, dtype=torch.uint8, device="cuda")
    from paper_2609_13692_gb300 import kv

    new = (spread * torch.randn((2, sum(kv_lens), kv_heads, dim), generator=gen, device="cuda")).to(BF16)
    every = torch.tensor(np.concatenate([[0], np.cumsum(kv_lens)]), dtype=torch.int32, device="cuda") if kv_lens else at
    kv.mpt_kv4_write(new[0], new[1], pages, table, every, lens)
    q = (1.5 * torch.randn((sum(q_lens), heads, dim), generator=gen, device="cuda")).to(dtype)
    return dict(q=q, pages=pages, table=table, at=at, lens=lens)


def args(c):
    return c["q"], c["pages"], c["table"], c["at"], c["lens"]


def check(kv, c, causal=True, hint=0, scale=None, **more):
    out, lse = kv.mpt_kv4_attend(*args(c), causal=causal, max_q_len=hint, scale=scale, **more)
    kv.mpt_kv_check()
    want, want_lse, tol, tol_lse = K.attend(*args(c), causal, scale or 1 / math.sqrt(c["q"].shape[2]))
    none = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse) & (lse < 0), none)
    assert bool((out[none] == 0).all())
    assert bool(((lse.double() - want_lse).abs()[~none] <= tol_lse[~none]).all())
    off = (out.double() - want).abs() - tol
    assert bool((off[~none] <= 0).all()), float(off[~none].max())
    return out, lse


# heads, kv_heads, dim: every number of groups of 32, groups of 1 to 40 heads
LAYOUTS = [(8, 8, 64), (8, 2, 128), (4, 1, 96), (9, 3, 80), (5, 1, 8), (16, 1, 128), (24, 1, 72), (6, 2, 256), (4, 4, 200),
           (40, 2, 128), (12, 1, 32), (3, 1, 160), (10, 1, 192), (33, 3, 56)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv_heads,dim", LAYOUTS)
def test_single_tokens(kv, heads, kv_heads, dim, dtype):
    check(kv, make(1, [1] * 9, [1, 2, 63, 64, 65, 130, 700, 1, 300], heads, kv_heads, dim, 16, dtype), hint=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim", LAYOUTS)
def test_chunks(kv, heads, kv_heads, dim, causal):
    check(kv, make(2, [1, 5, 0, 40, 129, 3, 257], [300, 5, 70, 200, 130, 1000, 257], heads, kv_heads, dim, 32, BF16), causal, hint=257)


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
def test_page_sizes(kv, page):
    check(kv, make(3, [1, 1, 7], [page - 1, 3 * page + 1, 515], 8, 4, 128, page, BF16))
    check(kv, make(4, [200, 31], [777, 31], 8, 4, 64, page, F16))
    check(kv, make(5, [40], [page + 41], 4, 2, 96, page, F16), hint=40)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_holes(kv, dim, causal):
    """Pages that the cache does not hold, at whole requests too; ids far out of range."""
    c = make(6, [1, 1, 3, 50, 200, 2], [100, 16, 400, 333, 1000, 64], 8, 2, dim, 16, BF16, holes=0.4)
    c["table"][1] = -1
    c["table"][5] = -1
    check(kv, c, causal)
    check(kv, c, causal, hint=200)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_that_see_nothing(kv, dim):
    """No keys at all; more new tokens than keys (the first stand before the cache's beginning)."""
    for hint in (0, 1, 300):
        check(kv, make(7, [1, 2, 300, 4, 129], [0, 0, 0, 1, 100], 4, 2, dim, 16, BF16), True, hint)
        check(kv, make(8, [1, 2, 300, 4], [0, 0, 5, 0], 4, 2, dim, 16, BF16), False, hint)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("q_lens", [[1, 1, 2], [130, 5, 40]])
def test_sizes_of_queries_and_values(kv, q_lens, dtype):
    """Rows of very large and very small elements, values near the largest that codes hold."""
    c = make(9, q_lens, [200, 70, 333], 8, 2, 128, 16, dtype, spread=700.0)
    big, small = (1e30, 1e-30) if dtype is BF16 else (1e3, 1e-7)
    c["q"][0] = (c["q"][0].float() * small).to(dtype)
    c["q"][1] = 0
    check(kv, c, hint=max(q_lens), scale=1e-5)
    c["q"][-1] = (c["q"][-1].float() * big).to(dtype)
    check(kv, c, hint=max(q_lens), scale=1e-35 if dtype is BF16 else 1e-9)


@pytest.mark.parametrize("q_lens", [[1], [3], [70]])
def test_long_keys_in_the_tail(kv, q_lens):
    """One key far above the rest, and many equal ones: small probabilities keep their weight."""
    c = make(10, q_lens, [20_001], 8, 2, 128, 64, F16)
    c["q"] *= 4
    check(kv, c, hint=max(q_lens))


@pytest.mark.parametrize("hint", [1, 600])
def test_many_requests(kv, hint):
    rng = random.Random(11)
    kv_lens = [rng.randint(0, 90) for _ in range(700)]
    check(kv, make(11, [rng.choice([0, 1, 1, 3]) for _ in kv_lens], kv_lens, 4, 2, 64, 8, BF16), hint=hint)


def test_rows_behind_the_last_request_and_strides(kv):
    c = make(12, [3, 50], [80, 200], 6, 2, 96, 16, BF16)
    want, want_lse = check(kv, c)
    for hint in (1, 50):
        wide = torch.full((60, 8, 104), 3.0, dtype=BF16, device="cuda")
        q = torch.zeros((60, 8, 104), dtype=BF16, device="cuda")
        q[:53, :6, :96] = c["q"]
        lse = torch.full((60, 6), 3.0, device="cuda")
        kv.mpt_kv4_attend(q[:, :6, :96], *args(c)[1:], max_q_len=hint, out=wide[:, :6, :96], lse=lse)
        kv.mpt_kv_check()
        assert bool((wide[53:] == 3).all()) and bool((wide[:, 6:] == 3).all()) and bool((wide[:, :, 96:] == 3).all())
        assert bool((lse[53:] == 3).all())
        assert bool(((wide[:53, :6, :96].float() - want.float()).abs() <= 2 ** -6 * (1 + want.float().abs())).all())
        assert bool(((lse[:53] - want_lse).abs() <= 1e-4).all())


def test_offsets_that_decrease_do_nothing(kv):
    c = make(13, [4, 4, 4], [50, 60, 70], 4, 2, 64, 16, BF16)
    c["at"] = torch.tensor([0, 8, 4, 12], dtype=torch.int32, device="cuda")
    for hint in (1, 100):
        out, lse = torch.full_like(c["q"], 7.0), torch.full((12, 4), 7.0, device="cuda")
        kv.mpt_kv4_attend(*args(c), max_q_len=hint, out=out, lse=lse)
        kv.mpt_kv_check()
        assert bool((out == 7).all()) and bool((lse == 7).all())


def test_same_bits_on_streams_and_in_graphs(kv):
    """Two streams at once with a workspace each, and a captured step (write, then attention) replayed
    with new inputs in the same buffers."""
    cases = [make(14, [1] * 20, [500 + 37 * i for i in range(20)], 8, 2, 128, 16, BF16), make(15, [100, 3], [700, 40], 8, 2, 128, 16, BF16)]
    want = [kv.mpt_kv4_attend(*args(c)) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for _ in range(3):
        for s, c in zip(streams, cases):
            got.append(kv.mpt_kv4_attend(*args(c), stream=s.cuda_stream))
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])

    c = cases[0]
    turns = torch.from_numpy(K.angles(2000, 128)).cuda()
    new = torch.randn((2, 20, 2, 128), device="cuda").to(BF16)
    q_in = c["q"].clone()
    space = torch.empty(kv.mpt_kv4_attend_workspace_bytes(), dtype=torch.uint8, device="cuda")

    def step():
        q = kv.mpt_kv4_write(new[0], new[1], c["pages"], c["table"], c["at"], c["lens"], rotation=turns, q=q_in)
        return kv.mpt_kv4_attend(q, *args(c)[1:], max_q_len=1, workspace=space)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    for seed in range(3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new.copy_(torch.randn(new.shape, generator=gen, device="cuda"))
        q_in.copy_(torch.randn(q_in.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        a, b = out.clone(), lse.clone()
        again = step()
        assert torch.equal(a, again[0]) and torch.equal(b, again[1])


def test_served_like_a_cache_in_16_bits(kv):
    """Prompts written and attended over in both caches: pages forked and copied as raw bytes, the same
    answers within what four bits lose."""
    gen = torch.Generator(device="cuda").manual_seed(16)
    page, heads, kv_heads, dim, n_pages = 16, 8, 2, 128, 40
    i32 = dict(dtype=torch.int32, device="cuda")
    size = kv.mpt_kv4_page_bytes(page, dim)
    pool = torch.zeros((1, n_pages, kv_heads, size), dtype=torch.uint8, device="cuda")
    wide = torch.zeros((1, n_pages, 2, page, kv_heads, dim), dtype=BF16, device="cuda")
    table, lens, refs = torch.full((3, 9), -1, **i32), torch.zeros(3, **i32), torch.zeros(n_pages, **i32)
    turns = torch.from_numpy(K.angles(200, dim)).cuda()

    def append(rows, at, k, v, q):
        a = kv.mpt_kv4_write(k, v, pool[0], table[rows], at, lens[rows], rotation=turns, q=q)
        b = kv.mpt_kv_write_rotated(k, v, turns, wide[0, :, 0], wide[0, :, 1], table[rows], at, lens[rows], q=q)
        assert torch.equal(a, b)
        return a

    kv.mpt_kv_extend(table, lens, refs, page, torch.zeros(1, **i32), torch.full((1,), 70, **i32))
    x = torch.randn((70, heads + 2 * kv_heads, dim), generator=gen, device="cuda").to(BF16)
    append(slice(0, 1), torch.tensor([0, 70], **i32), x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], x[:, :heads])
    old, fresh, _ = kv.mpt_kv_fork(table, lens, refs, page, torch.zeros(2, **i32), torch.tensor([1, 2], **i32), torch.full((2,), 70, **i32))
    kv.mpt_kv_copy_pages(pool, old, fresh)
    kv.mpt_kv_copy_pages(wide, old, fresh)
    kv.mpt_kv_extend(table, lens, refs, page, torch.tensor([1, 2], **i32), torch.tensor([1, 40], **i32))
    at = torch.tensor([0, 1, 41], **i32)
    x = torch.randn((41, heads + 2 * kv_heads, dim), generator=gen, device="cuda").to(BF16)
    q = append(slice(1, 3), at, x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], x[:, :heads])
    out, lse = kv.mpt_kv4_attend(q, pool[0], table[1:], at, lens[1:], max_q_len=40)
    ref, ref_lse = kv.mpt_kv_attend(q, wide[0, :, 0], wide[0, :, 1], table[1:], at, lens[1:], max_q_len=40)
    kv.mpt_kv_check()
    # a step of a group of 32 normal values is about 4.2 / 15, its error evenly spread: 0.08 a value
    assert float((out.float() - ref.float()).norm() / ref.float().norm()) < 0.2
    assert float((lse - ref_lse).abs().max()) < 0.5
    k, v = kv.mpt_kv4_read(pool[0], table[1:], at, lens[1:], 41, dim)
    assert float((v.float() - x[:, heads + kv_heads:].float()).norm() / v.float().norm()) < 0.12
    want, want_lse, tol, tol_lse = K.attend(q, pool[0], table[1:], at, lens[1:], True, 1 / math.sqrt(dim))
    assert bool(((out.double() - want).abs() <= tol).all())
