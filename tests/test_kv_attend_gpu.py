"""mpt_kv_attend against attention in 64 bits: types, head layouts, lengths from none to long, odd head
sizes, strides, pages that end inside a tile, holes, rows that see nothing, and NaN in masked places."""

import math
import random

import pytest

torch = pytest.importorskip("torch")

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


def make(seed, q_lens, kv_lens, heads, kv_heads, dim, page, dtype, order="token", holes=0.0, spare=3, poison=False,
         table_pad=0):
    """A cache with its pages in random order; with `poison`, NaN wherever nothing is stored."""
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in kv_lens]
    n_pages, width = sum(need) + spare, max([1, *need]) + 1
    shape = (n_pages, 2, page, kv_heads, dim) if order == "token" else (n_pages, 2, kv_heads, page, dim)
    pool = torch.randn(shape, generator=gen, device="cuda").to(dtype)
    k, v = pool[:, 0], pool[:, 1]
    if order == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    ids = list(range(n_pages))
    rng.shuffle(ids)
    table = torch.full((len(kv_lens), width + table_pad), n_pages + 5 if poison else -1, dtype=torch.int32)
    stored = torch.zeros((n_pages, page), dtype=torch.bool)
    for i, n in enumerate(need):
        for t in range(n):
            p = ids.pop()
            stored[p, :min(page, kv_lens[i] - t * page)] = True
            if rng.random() < holes:
                p = rng.choice([-1, n_pages, -2 ** 31, 2 ** 31 - 1])
            table[i, t] = p
    if poison:
        k[~stored.cuda()] = math.nan
        v[~stored.cuda()] = math.nan
    at = [0]
    for n in q_lens:
        at.append(at[-1] + n)
    q = (1.5 * torch.randn((at[-1], heads, dim), generator=gen, device="cuda")).to(dtype)
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(q=q, k=k, v=v, table=table.cuda()[:, :width], at=torch.tensor(at, **i32), lens=torch.tensor(kv_lens, **i32))


def args(c):
    return c["q"], c["k"], c["v"], c["table"], c["at"], c["lens"]


def check(kv, c, causal=True, hint=0, scale=None, **more):
    out, lse = kv.mpt_kv_attend(*args(c), causal=causal, max_q_len=hint, scale=scale, **more)
    kv.mpt_kv_check()
    want, want_lse, tol, tol_lse = M.attend(*args(c), causal, scale or 1 / math.sqrt(c["q"].shape[2]))
    none = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse) & (lse < 0), none)
    assert bool((out[none] == 0).all())
    assert bool(((lse.double() - want_lse).abs()[~none] <= tol_lse[~none]).all())
    off = (out.double() - want).abs() - tol
    assert bool((off[~none] <= 0).all()), float(off[~none].max())
    return out, lse


# heads, kv_heads, dim
LAYOUTS = [(8, 8, 64), (8, 2, 128), (4, 1, 96), (9, 3, 80), (5, 1, 8), (16, 1, 128), (24, 1, 72), (6, 2, 256), (4, 4, 200),
           (40, 2, 128)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv_heads,dim", LAYOUTS)
def test_single_tokens(kv, heads, kv_heads, dim, dtype):
    kv_lens = [1, 2, 63, 64, 65, 130, 700, 1, 300]
    check(kv, make(1, [1] * 9, kv_lens, heads, kv_heads, dim, 16, dtype, poison=True), hint=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim", LAYOUTS)
def test_chunks(kv, heads, kv_heads, dim, causal):
    q_lens = [1, 5, 0, 40, 129, 3, 257]
    kv_lens = [300, 5, 70, 200, 130, 1000, 257]
    check(kv, make(2, q_lens, kv_lens, heads, kv_heads, dim, 32, BF16, poison=True), causal, hint=257)


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
def test_page_sizes(kv, page, order):
    check(kv, make(3, [1, 1, 7], [page - 1, 3 * page + 1, 515], 8, 4, 128, page, BF16, order, poison=True))
    check(kv, make(4, [200, 31], [777, 31], 8, 4, 64, page, F16, order, poison=True))
    check(kv, make(5, [40], [page + 41], 4, 2, 128, page, F16, order, poison=True), hint=40)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_holes(kv, dim, causal):
    """Pages that the cache does not hold, at whole requests too; ids far out of range."""
    c = make(6, [1, 1, 3, 50, 200, 2], [100, 16, 400, 333, 1000, 64], 8, 2, dim, 16, BF16, holes=0.4, poison=True)
    c["table"][1] = -1
    c["table"][5] = -1
    check(kv, c, causal)
    check(kv, c, causal, hint=200)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_that_see_nothing(kv, dim):
    """No keys at all; more new tokens than keys (the first stand before the cache's beginning)."""
    for hint in (0, 1, 300):
        check(kv, make(7, [1, 2, 300, 4, 129], [0, 0, 0, 1, 100], 4, 2, dim, 16, BF16, poison=True), True, hint)
        check(kv, make(8, [1, 2, 300, 4], [0, 0, 5, 0], 4, 2, dim, 16, BF16, poison=True), False, hint)


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (4, 4, 64), (2, 1, 256), (6, 2, 96)])
def test_masked_values_that_are_not_finite(kv, heads, kv_heads, dim):
    """A later token's NaN or infinite key and value leave the rows before it alone, and reach those after it."""
    q_lens, kv_lens = [4, 70, 300, 2], [100, 200, 300, 64]
    for dtype in (BF16, F16):
        c = make(9, q_lens, kv_lens, heads, kv_heads, dim, 16, dtype, poison=True)
        clean, _ = check(kv, c)
        hit = [98, 170, 150, 63]
        first = [0, 4, 74, 374]
        for i, j in enumerate(hit):
            page = int(c["table"][i, j // 16])
            c["k"][page, j % 16] = math.nan if i % 2 else math.inf
            c["v"][page, j % 16] = -math.inf if i % 2 else math.nan
        out, lse = kv.mpt_kv_attend(*args(c))
        kv.mpt_kv_check()
        want, _, tol, _ = M.attend(*args(make(9, q_lens, kv_lens, heads, kv_heads, dim, 16, dtype)), True, 1 / math.sqrt(dim))
        for i, j in enumerate(hit):
            before = j - (kv_lens[i] - q_lens[i])  # tokens of the chunk that stand before key j
            a, b = first[i], first[i] + before
            assert bool(torch.isfinite(out[a:b]).all()) and bool(torch.isfinite(lse[a:b]).all())
            assert bool(((out[a:b].double() - want[a:b]).abs() <= tol[a:b]).all())
            assert bool(torch.isnan(out[b:first[i] + q_lens[i]]).any(-1).all())


def test_infinite_value_that_is_seen(kv):
    """A visible infinity comes through, beside masked NaN in the same tile."""
    c = make(10, [3], [40], 2, 1, 64, 8, BF16, poison=True)
    page = int(c["table"][0, 37 // 8])
    c["v"][page, 37 % 8, 0, 5] = math.inf
    out, _ = kv.mpt_kv_attend(*args(c))
    assert bool(torch.isposinf(out[:, :, 5]).all())
    out[:, :, 5] = 0
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_far_scores(kv, dim):
    """Scores of hundreds, and keys that all but one token outweigh: nothing overflows."""
    for big in (30.0, 300.0):
        c = make(11, [1, 20, 150], [513, 700, 150], 4, 2, dim, 16, BF16)
        c["q"].mul_(big)
        out, lse = kv.mpt_kv_attend(*args(c))
        want, want_lse, tol, tol_lse = M.attend(*args(c), True, 1 / math.sqrt(dim))
        assert bool(((out.double() - want).abs() <= tol).all())
        assert bool(((lse.double() - want_lse).abs() <= tol_lse).all())


@pytest.mark.parametrize("dim", [64, 128, 96])
def test_strides(kv, dim):
    """q and out as views of wider tensors, a wider table, an own scale, given outputs and workspace."""
    for q_lens in ([1, 1, 1], [30, 1, 200]):
        c = make(12, q_lens, [77, 500, 250], 6, 2, dim, 16, BF16, table_pad=13)
        wide = torch.zeros((c["q"].shape[0], 3, 8, dim + 8), dtype=BF16, device="cuda")
        view = wide[:, 1, 1:7, :dim]
        view.copy_(c["q"])
        c["q"] = view
        room = torch.full((view.shape[0], 9, dim + 16), 7.0, dtype=BF16, device="cuda")
        out = room[:, 2:8, 8:dim + 8]
        lse = torch.empty(view.shape[:2], device="cuda")
        ws = torch.empty(kv.mpt_kv_attend_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
        check(kv, c, scale=0.07, out=out, lse=lse, workspace=ws)
        room[:, 2:8, 8:dim + 8] = 7.0
        assert bool((room == 7.0).all())


def test_many_requests(kv):
    rng = random.Random(5)
    kv_lens = [rng.choice([0, 1, 2, 9, 40]) for _ in range(1500)]
    check(kv, make(13, [1] * 1500, kv_lens, 4, 2, 64, 8, BF16, poison=True))
    q_lens = [rng.choice([0, 0, 1, 3]) for _ in range(1200)]
    check(kv, make(14, q_lens, [n + 5 for n in q_lens], 4, 2, 128, 8, F16, poison=True))


@pytest.mark.parametrize("dim", [64, 128])
def test_more_items_than_a_block_lists(kv, dim):
    """Thousands of small items, whole and cut, in both kernels."""
    rng = random.Random(6)
    q_lens = [rng.choice([0, 1, 2, 5, 70]) for _ in range(900)]
    kv_lens = [n + rng.choice([0, 1, 30, 200]) for n in q_lens]
    c = make(22, q_lens, kv_lens, 8, 8, dim, 8, BF16, poison=True)
    check(kv, c, hint=70)
    check(kv, c, hint=1)


@pytest.mark.parametrize("q_len,heads", [(1, 8), (1, 64), (33, 8), (300, 2)])
def test_long_keys(kv, q_len, heads):
    """Few rows over many keys: the keys are cut across all blocks and joined."""
    check(kv, make(15, [q_len], [20_011], heads, 2, 128, 16, BF16, poison=True), hint=q_len)
    check(kv, make(16, [q_len, 0, q_len], [9_000, 12, 5_003], heads, 1, 64, 64, F16, poison=True), False)


@pytest.mark.parametrize("q_len", [1, 33])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 256), (6, 2, 96), (3, 3, 200)])
def test_long_keys_of_other_heads(kv, heads, kv_heads, dim, q_len):
    """Many turns of the rings of copies, with requests of other lengths beside."""
    c = make(23, [q_len, 1, q_len], [12_345, 700, 4_100], heads, kv_heads, dim, 16, BF16, poison=True)
    check(kv, c, hint=q_len)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scores_that_grow_along_the_keys(kv, dim, causal):
    """The running maximum is outgrown in tile after tile, the last among them."""
    for q_lens, kv_lens in (([1, 3], [1_500, 640]), ([150, 40, 300], [1_500, 641, 300])):
        c = make(24, q_lens, kv_lens, 4, 2, dim, 16, BF16)
        lead = torch.randn(dim, device="cuda").to(BF16)
        c["q"].copy_(lead.expand_as(c["q"]) * (1 + 0.1 * torch.rand(c["q"].shape[:2], device="cuda"))[..., None])
        for i, n in enumerate(kv_lens):
            j = torch.arange(n, device="cuda")
            c["k"][c["table"][i].long()[j // 16], j % 16] += ((j // 100).float() * 0.2)[:, None, None].to(BF16) * lead
        check(kv, c, causal, hint=max(q_lens))


def test_offsets_beyond_32_bits(kv):
    """Pages whose elements lie past 2^31 and 2^32."""
    n_pages, page, kv_heads, dim = 70_000, 64, 8, 128
    pool = torch.empty((n_pages, page, kv_heads, dim), dtype=BF16, device="cuda")
    far = [n_pages - 1, 40_000, 66_000, 3]
    pool[far] = torch.randn((4, page, kv_heads, dim), device="cuda").to(BF16)
    i32 = dict(dtype=torch.int32, device="cuda")
    for q_len in (1, 130):
        c = dict(q=torch.randn((q_len, 16, dim), device="cuda").to(BF16), k=pool, v=pool,
                 table=torch.tensor([far], **i32), at=torch.tensor([0, q_len], **i32), lens=torch.tensor([250], **i32))
        check(kv, c, hint=q_len)


def test_lengths_out_of_range_are_clamped(kv):
    """Lengths beyond the table, negative ones and offsets beyond the tokens stay inside the tensors."""
    c = make(17, [1, 1, 4], [50, 60, 70], 4, 2, 64, 16, BF16)
    c["lens"] = torch.tensor([10 ** 9, -5, 70], dtype=torch.int32, device="cuda")
    c["at"] = torch.tensor([0, 1, 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out, lse = kv.mpt_kv_attend(*args(c))
    kv.mpt_kv_check()
    assert bool(torch.isneginf(lse[1]).all())
    c["at"] = torch.tensor([3, -7, 100, 1], dtype=torch.int32, device="cuda")
    kv.mpt_kv_attend(*args(c))
    kv.mpt_kv_check()


def test_hints_and_repeats_give_the_same(kv):
    c = make(18, [1, 3, 1, 1], [5000, 700, 64, 3], 8, 2, 128, 16, BF16)
    a = kv.mpt_kv_attend(*args(c))
    b = kv.mpt_kv_attend(*args(c))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for hint in (1, 3, 10_000):
        check(kv, c, hint=hint)


def test_streams_and_graphs(kv):
    """Calls on a stream of the caller's, and captured in a graph whose replay reads new lengths."""
    c = make(19, [1, 40], [300, 500], 8, 2, 128, 16, BF16)
    want = kv.mpt_kv_attend(*args(c))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = kv.mpt_kv_attend(*args(c), stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = kv.mpt_kv_attend(*args(c))
    c["lens"].copy_(torch.tensor([17, 444], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    want = kv.mpt_kv_attend(*args(c))
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_empty(kv):
    c = make(20, [1], [10], 4, 2, 64, 16, BF16)
    i32 = dict(dtype=torch.int32, device="cuda")
    none = dict(c, q=c["q"][:0], at=torch.zeros(2, **i32))
    out, lse = kv.mpt_kv_attend(*args(none))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    none = dict(c, q=c["q"][:0], at=torch.zeros(1, **i32), lens=c["lens"][:0], table=c["table"][:0])
    assert kv.mpt_kv_attend(*args(none))[0].shape == (0, 4, 64)


def test_refusals(kv):
    from paper_2609_13692_gb300.mpt import MPTError

    c = make(21, [1, 1], [40, 30], 4, 2, 64, 16, BF16)

    def status(**more):
        with pytest.raises(MPTError) as e:
            kv.mpt_kv_attend(*args({**c, **{k: v for k, v in more.items() if k in c}}),
                             **{k: v for k, v in more.items() if k not in c})
        return e.value.status

    assert status(scale=0.0) == 1 and status(scale=-1.0) == 1 and status(scale=math.nan) == 1 and status(scale=math.inf) == 1
    assert status(max_q_len=-1) == 1
    assert status(q=torch.zeros((2, 3, 64), dtype=BF16, device="cuda")) == 1        # 3 heads over 2
    assert status(q=torch.zeros((2, 258, 64), dtype=BF16, device="cuda")) == 2      # group of 129
    assert status(q=torch.zeros((2, 4, 65), dtype=BF16, device="cuda")[:, :, :64]) == 1   # stride of 65
    assert status(q=torch.zeros((2, 4, 72), dtype=BF16, device="cuda")[:, :, 1:65]) == 1  # not 16-byte aligned
    assert status(workspace=torch.empty(64, dtype=torch.uint8, device="cuda")) == 5
    bad = torch.zeros((4, 12, 2, 64), dtype=BF16, device="cuda")
    assert status(k=bad, v=bad) == 1                                                # pages of 12
    bad = torch.zeros((4, 512, 2, 64), dtype=BF16, device="cuda")
    assert status(k=bad, v=bad) == 1                                                # pages of 512
    bad = torch.zeros((4, 16, 2, 264), dtype=BF16, device="cuda")
    assert status(k=bad, v=bad, q=torch.zeros((2, 4, 264), dtype=BF16, device="cuda")) in (1, 2)
    bad = torch.zeros((4, 16, 2, 60), dtype=BF16, device="cuda")
    assert status(k=bad, v=bad, q=torch.zeros((2, 4, 60), dtype=BF16, device="cuda")) == 1
    for more in (dict(q=c["q"].float()), dict(q=c["q"].half()), dict(lens=c["lens"].long()), dict(at=c["at"][:2]),
                 dict(k=c["k"].float(), v=c["v"].float()), dict(q=c["q"].cpu()), dict(q=c["q"][0]),
                 dict(q=c["q"].transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            kv.mpt_kv_attend(*args({**c, **more}))
    with pytest.raises(ValueError):
        kv.mpt_kv_attend(*args(c), out=torch.empty((2, 4, 64), device="cuda"))
    with pytest.raises(ValueError):
        kv.mpt_kv_attend(*args(c), lse=torch.empty((4, 2), device="cuda"))
