"""Edges of the turned writes and of the cache in 4 bits: every step of a group, sizes at their limits,
scores far apart, offsets beyond 32 bits, lengths out of range, many requests and items, gradients."""

import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import kv4_model as K
from tests.test_kv4_gpu import BF16, F16, args, check, kv, make  # noqa: F401

pytestmark = pytest.mark.gpu


def test_every_step(kv):  # noqa: F811
    """Groups whose range or largest value asks for each step that a byte can hold, at it and beside it:
    ranges on the border between two steps, values on the border between two codes."""
    rows = []
    for e in range(-20, 10):
        for m in range(8, 16):
            s = m / 8 * 2.0 ** e
            for off, near in ((0, 0), (-7, 0), (3, 0), (-120, 0), (105, 0), (0, 1), (-8, 1), (0, -1)):
                g = (off + np.arange(32) % 16 + 0.5 * (np.arange(32) % 3 == 0) * (np.arange(32) < 16)) * s
                g[0], g[1] = off * s, (off + 15) * s
                rows.append(np.nextafter(g.astype(np.float32), np.float32(near * 1e30)) if near else g)
    x = torch.from_numpy(np.array(rows, dtype=np.float32))
    i32 = dict(dtype=torch.int32, device="cuda")
    for dtype in (BF16, F16):
        new = x.clamp(-60000, 60000).to(dtype)[:, None].cuda()
        n = len(new)
        pages = torch.zeros((-(-n // 256), 1, kv.mpt_kv4_page_bytes(256, 32)), dtype=torch.uint8, device="cuda")
        table = torch.arange(len(pages), **i32)[None]
        kv.mpt_kv4_write(new, new, pages, table, torch.tensor([0, n], **i32), torch.tensor([n], **i32))
        kv.mpt_kv_check()
        want = np.zeros(pages.shape, dtype=np.uint8)
        f = new.float().cpu().numpy()[:, 0]
        for t in range(n):
            K.put(want, 32, t // 256, t % 256, 0, f[t], f[t])
        assert np.array_equal(pages.cpu().numpy(), want)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page,dim,q_len,rest", [(32, 64, 1, 32), (256, 128, 3, 200), (32, 128, 40, 27), (16, 128, 2, 16), (8, 256, 50, 5)])
def test_keys_up_to_the_last_of_32_bits(kv, page, dim, q_len, rest, causal):  # noqa: F811
    """A sparse table as wide as it may be, its last page beside 2^31: new tokens written there and read
    back, and the keys that are there, as a cache of their own."""
    width = (2 ** 31 - 1) // page
    gen = torch.Generator(device="cuda").manual_seed(page)
    pages = torch.randint(0, 256, (7, 2, kv.mpt_kv4_page_bytes(page, dim)), generator=gen, dtype=torch.uint8, device="cuda")
    pages.copy_(pages & 0x7F)  # steps of ordinary size
    i32 = dict(dtype=torch.int32, device="cuda")
    near = -(-q_len // page) + 1  # the pages of the new tokens, one more
    table = torch.full((1, width), -1, **i32)
    there = [0, 12_345_678 // page, *range(width - near, width)]
    ids = [3, 6, *([1, 0, 2, 4, 1, 0, 2] * 2)[:near - 1], 5]
    table[0, torch.tensor(there, device="cuda")] = torch.tensor(ids, **i32)
    at, lens = torch.tensor([0, q_len], **i32), (width - 1) * page + rest
    assert lens > 2 ** 31 - 2 * page
    q = torch.randn((q_len, 4, dim), generator=gen, device="cuda").to(BF16) * 2.0 ** -4
    new = torch.randn((2, q_len, 2, dim), generator=gen, device="cuda").to(BF16)
    kv.mpt_kv4_write(new[0], new[1], pages, table, at, torch.tensor([lens], **i32))
    out, lse = kv.mpt_kv4_attend(q, pages, table, at, torch.tensor([lens], **i32), causal=causal, max_q_len=q_len)
    k, v = kv.mpt_kv4_read(pages, table, at, torch.tensor([lens], **i32), q_len, dim, dtype=torch.float32)
    kv.mpt_kv_check()
    few = torch.tensor([ids], **i32), at, torch.tensor([(len(ids) - 1) * page + rest], **i32)
    vals = K.values(pages, dim)
    j = torch.arange(q_len) + int(few[2][0]) - q_len
    for got, x in zip((k, v), vals):
        assert torch.equal(got, x[few[0][0].long().cpu()[j // page], j % page])
    want, want_lse, tol, tol_lse = K.attend(q, pages, *few, causal, 1 / math.sqrt(dim))
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - want_lse).abs() <= tol_lse).all())


def test_offsets_beyond_32_bits(kv):  # noqa: F811
    """Pages whose bytes lie past 2^32: written, read and attended over; those between are left alone."""
    page, kv_heads, dim = 256, 8, 256
    size = kv.mpt_kv4_page_bytes(page, dim)
    n_pages = (9 << 30) // (kv_heads * size)
    pages = torch.empty((n_pages, kv_heads, size), dtype=torch.uint8, device="cuda")
    far = [n_pages - 1, n_pages // 2, 3, n_pages - 7]
    assert far[1] * kv_heads * size > 2 ** 32
    pages[[i - 1 for i in far]] = 9
    i32 = dict(dtype=torch.int32, device="cuda")
    table, lens, n = torch.tensor([far], **i32), torch.tensor([1000], **i32), 1000
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = torch.randn((2, n, kv_heads, dim), generator=gen, device="cuda").to(BF16)
    turns = torch.from_numpy(K.angles(1000, dim)).cuda()
    kv.mpt_kv4_write(new[0], new[1], pages, table, torch.tensor([0, n], **i32), lens, rotation=turns)
    assert bool((pages[[i - 1 for i in far]] == 9).all())
    held = pages[far]
    near = torch.arange(4, **i32)[None]
    for q_len in (1, 130):
        at = torch.tensor([0, q_len], **i32)
        q = torch.randn((q_len, 16, dim), generator=gen, device="cuda").to(BF16)
        got = kv.mpt_kv4_attend(q, pages, table, at, lens, max_q_len=q_len)
        same = kv.mpt_kv4_attend(q, held, near, at, lens, max_q_len=q_len)
        assert torch.equal(got[0], same[0]) and torch.equal(got[1], same[1])
        assert all(torch.equal(a, b) for a, b in zip(kv.mpt_kv4_read(pages, table, at, lens, q_len, dim), kv.mpt_kv4_read(held, near, at, lens, q_len, dim)))
    want, want_lse, tol, tol_lse = K.attend(q, held, near, at, lens, True, 1 / math.sqrt(dim))
    kv.mpt_kv_check()
    assert bool(((same[0].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("hint", [1, 40])
def test_lengths_out_of_range_are_clamped(kv, hint):  # noqa: F811
    """Negative lengths, lengths beyond the table, offsets beyond the tokens: as the clamped ones."""
    c = make(21, [1, 40, 3, 5], [60, 64, 9, 30], 4, 2, 64, 16, BF16)
    cap = c["table"].shape[1] * 16
    for lens, same in (([60, 2 ** 31 - 1, -5, -2 ** 31], [60, cap, 0, 0]),):
        out, lse = kv.mpt_kv4_attend(*args(c)[:4], torch.tensor(lens, dtype=torch.int32, device="cuda"), max_q_len=hint)
        want, want_lse = kv.mpt_kv4_attend(*args(c)[:4], torch.tensor(same, dtype=torch.int32, device="cuda"), max_q_len=hint)
        kv.mpt_kv_check()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    at = torch.tensor([0, 1, 41, 44, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out, _ = kv.mpt_kv4_attend(c["q"], c["pages"], c["table"], at, c["lens"], max_q_len=hint)
    new = torch.ones((49, 2, 64), dtype=BF16, device="cuda")
    before = c["pages"].clone()
    kv.mpt_kv4_write(new, new, c["pages"], c["table"], at, torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, 3], dtype=torch.int32, device="cuda"))
    kv.mpt_kv_check()
    assert torch.equal(c["pages"], before)  # every position is outside the table


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_far_scores(kv, dim):  # noqa: F811
    """Scores of hundreds, and keys that all but one token outweigh: nothing overflows."""
    for big in (30.0, 300.0):
        c = make(22, [1, 20, 150], [513, 700, 150], 4, 2, dim, 16, BF16)
        c["q"].mul_(big)
        check(kv, c)
        check(kv, c, hint=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128, 160, 256])
def test_scores_that_grow_along_the_keys(kv, dim, causal):  # noqa: F811
    """The running maximum is outgrown in tile after tile, the last among them."""
    for q_lens, kv_lens in (([1, 3], [1_500, 640]), ([150, 40, 300], [1_500, 641, 300])):
        c = make(23, q_lens, kv_lens, 4, 2, dim, 16, BF16)
        lead = torch.randn(dim, device="cuda")
        c["q"].copy_(lead.expand(c["q"].shape) * (1 + 0.1 * torch.rand(c["q"].shape[:2], device="cuda"))[..., None])
        j = torch.cat([torch.arange(n, device="cuda") for n in kv_lens])
        k = torch.randn((len(j), 2, dim), device="cuda") + ((j // 100).float() * 0.2)[:, None, None] * lead
        every = torch.tensor([0, *np.cumsum(kv_lens)], dtype=torch.int32, device="cuda")
        kv.mpt_kv4_write(k.to(BF16), torch.randn_like(k).to(BF16), c["pages"], c["table"], every, c["lens"])
        check(kv, c, causal, hint=max(q_lens))


@pytest.mark.parametrize("dim", [64, 128])
def test_more_items_than_a_block_lists(kv, dim):  # noqa: F811
    """Thousands of small items, whole and cut, in both kernels."""
    rng = random.Random(6)
    q_lens = [rng.choice([0, 1, 2, 5, 70]) for _ in range(900)]
    kv_lens = [n + rng.choice([0, 1, 30, 200]) for n in q_lens]
    c = make(24, q_lens, kv_lens, 8, 8, dim, 8, BF16)
    check(kv, c, hint=70)
    check(kv, c, hint=1)


@pytest.mark.parametrize("q_len,heads", [(1, 8), (1, 64), (33, 8), (300, 2)])
def test_long_keys(kv, q_len, heads):  # noqa: F811
    """Few rows over many keys: the keys are cut across all blocks and joined."""
    check(kv, make(25, [q_len], [20_011], heads, 2, 128, 16, BF16), hint=q_len)
    check(kv, make(26, [q_len, 0, q_len], [9_000, 12, 5_003], heads, 1, 64, 64, F16), False)


@pytest.mark.parametrize("q_len", [1, 33])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 256), (6, 2, 96), (3, 3, 200), (12, 1, 32)])
def test_long_keys_of_other_heads(kv, heads, kv_heads, dim, q_len):  # noqa: F811
    """Many turns of the rings, with requests of other lengths beside."""
    check(kv, make(27, [q_len, 1, q_len], [12_345, 700, 4_100], heads, kv_heads, dim, 16, BF16), hint=q_len)


@pytest.mark.parametrize("heads,kv_heads,dim", [(82, 2, 64), (43, 1, 256), (65, 1, 128), (200, 2, 96), (128, 1, 128), (128, 1, 200)])
def test_large_groups(kv, heads, kv_heads, dim):  # noqa: F811
    """41 to 128 query heads of a KV head: row tiles of three, two and one whole tokens."""
    for causal in (True, False):
        check(kv, make(28, [1, 1, 0, 1], [300, 1, 5, 130], heads, kv_heads, dim, 16, BF16), causal, hint=1)
        check(kv, make(29, [1, 7, 2, 30], [64, 7, 1, 257], heads, kv_heads, dim, 32, F16, holes=0.2), causal, hint=30)


def test_chunks_of_more_requests_than_the_large_kernel_lists(kv):  # noqa: F811
    """Above 8,192 requests the small kernel takes chunks too."""
    rng = random.Random(30)
    q_lens = [rng.choice([1, 3, 17, 70]) if i % 41 == 0 else 0 for i in range(8_200)]
    kv_lens = [max(0, n + rng.choice([-2, 0, 9, 150])) if n else i % 2 for i, n in enumerate(q_lens)]
    for dim, dtype in ((64, BF16), (256, F16)):
        check(kv, make(30, q_lens, kv_lens, 4, 2, dim, 16, dtype), hint=70)


@pytest.mark.parametrize("heads,dim", [(8, 128), (6, 96)])
def test_any_hint_gives_the_same(kv, heads, dim):  # noqa: F811
    """The hint chooses the kernel and the rows of an item; a wrong one costs time only."""
    c = make(31, [1, 9, 60], [100, 500, 61], heads, 2, dim, 16, BF16)
    for hint in (0, 1, 2, 4, 60, 10_000):
        check(kv, c, hint=hint)


def test_not_finite_queries(kv):  # noqa: F811
    """NaN and infinite queries stay in their rows."""
    for q_lens in ([1, 1, 1], [5, 70, 3]):
        c = make(32, q_lens, [50, 90, 300], 8, 2, 128, 16, BF16)
        clean, clean_lse = kv.mpt_kv4_attend(*args(c), max_q_len=max(q_lens))
        c["q"][0, 1, 5] = math.nan
        c["q"][-1, 6, 7] = math.inf
        out, lse = kv.mpt_kv4_attend(*args(c), max_q_len=max(q_lens))
        kv.mpt_kv_check()
        hit = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
        hit[0, 1] = hit[-1, 6] = True
        assert bool(out[hit].isnan().all())
        assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


def test_nothing_to_do(kv):  # noqa: F811
    c = make(33, [1, 2], [30, 40], 4, 2, 64, 16, BF16)
    none = torch.zeros((0, 3), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    before = c["pages"].clone()
    out, lse = kv.mpt_kv4_attend(c["q"][:0], c["pages"], c["table"], torch.zeros_like(c["at"]), c["lens"])
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    kv.mpt_kv4_attend(c["q"], c["pages"], *none)
    new = torch.ones((3, 2, 64), dtype=BF16, device="cuda")
    kv.mpt_kv4_write(new, new, c["pages"], *none)
    kv.mpt_kv4_write(new[:0], new[:0], c["pages"], c["table"], torch.zeros_like(c["at"]), c["lens"])
    assert kv.mpt_kv4_read(c["pages"], c["table"], torch.zeros_like(c["at"]), c["lens"], 0, 64)[0].shape == (0, 2, 64)
    kv.mpt_kv_check()
    assert torch.equal(c["pages"], before)


def test_refusals_and_gradients(kv):  # noqa: F811
    """What the binding turns down on a GPU; tensors that require gradients, but where none are recorded."""
    c = make(34, [1, 40], [30, 70], 4, 2, 64, 16, BF16)
    out, lse = kv.mpt_kv4_attend(*args(c))
    new = torch.ones((41, 2, 64), dtype=BF16, device="cuda")
    turns = torch.from_numpy(K.angles(70, 64)).cuda()
    pool = torch.zeros((9, 2, 16, 2, 64), dtype=BF16, device="cuda")
    where = args(c)[2:]
    small = torch.empty(256, dtype=torch.uint8, device="cuda")

    def req(t):
        return t.detach().clone().requires_grad_()

    for call in (lambda: kv.mpt_kv4_attend(req(c["q"]), *args(c)[1:]), lambda: kv.mpt_kv4_attend(*args(c), out=req(out)),
                 lambda: kv.mpt_kv4_write(req(new), new, c["pages"], *where), lambda: kv.mpt_kv4_write(new, req(new), c["pages"], *where),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=req(turns)),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=turns, q=req(c["q"])),
                 lambda: kv.mpt_kv4_read(c["pages"], *where, 41, 64, k_out=req(new)),
                 lambda: kv.mpt_kv_write_rotated(req(new), new, turns, pool[:, 0], pool[:, 1], *where),
                 lambda: kv.mpt_kv_write_rotated(new, new, turns, req(pool)[:, 0], pool[:, 1], *where),
                 lambda: kv.mpt_kv_write_rotated(new, new, turns, pool[:, 0], pool[:, 1], *where, q=req(c["q"]))):
        with pytest.raises(ValueError, match="no backward"):
            call()
    with torch.no_grad():
        assert torch.equal(kv.mpt_kv4_attend(req(c["q"]), *args(c)[1:])[0], out)
    for call in (lambda: kv.mpt_kv4_attend(c["q"].float(), *args(c)[1:]), lambda: kv.mpt_kv4_attend(c["q"], c["pages"].int(), *where),
                 lambda: kv.mpt_kv4_attend(c["q"][:, :, :40], c["pages"][:, :, :100], *where), lambda: kv.mpt_kv4_attend(*args(c), out=out[:1]),
                 lambda: kv.mpt_kv4_attend(*args(c), lse=lse.half()), lambda: kv.mpt_kv4_attend(c["q"], c["pages"].cpu(), *where),
                 lambda: kv.mpt_kv4_write(new, new.half(), c["pages"], *where), lambda: kv.mpt_kv4_write(new[:, :1], new[:, :1], c["pages"], *where),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, q=c["q"]),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=turns.double()),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=turns, q=c["q"][:3]),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=turns, positions=where[1]),
                 lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=turns, q_out=c["q"]),
                 lambda: kv.mpt_kv4_read(c["pages"], *where, 41, 64, dtype=torch.float64),
                 lambda: kv.mpt_kv4_read(c["pages"], *where, 41, 64, k_out=new[:3]),
                 lambda: kv.mpt_kv_write_rotated(new.half(), new.half(), turns, pool[:, 0], pool[:, 1], *where)):
        with pytest.raises(ValueError):
            call()
    from paper_2609_13692_gb300 import mpt

    for call, status in ((lambda: kv.mpt_kv4_attend(*args(c), workspace=small), None), (lambda: kv.mpt_kv4_attend(*args(c), scale=-1.0), 1),
                         (lambda: kv.mpt_kv4_write(new, new, c["pages"], *where, rotation=turns[:, :24]), 1),
                         (lambda: kv.mpt_kv4_attend(c["q"][:, :3], *args(c)[1:]), 1)):
        with pytest.raises(mpt.MPTError) as e:
            call()
        assert status is None or e.value.status == status


def test_heads_before_tokens_and_packed_queries(kv):  # noqa: F811
    """Pages as a view with heads first, queries of one packed tensor, outputs by heads."""
    c = make(35, [3, 50], [80, 200], 6, 2, 96, 16, BF16)
    for hint in (1, 50):
        want, want_lse = check(kv, c, hint=hint)
        by_head = c["pages"].transpose(0, 1).contiguous().transpose(0, 1)
        packed = torch.zeros((53, 10, 96), dtype=BF16, device="cuda")
        packed[:, 2:8] = c["q"]
        out = torch.empty((6, 53, 96), dtype=BF16, device="cuda").transpose(0, 1)
        got, lse = kv.mpt_kv4_attend(packed[:, 2:8], by_head, *args(c)[2:], max_q_len=hint, out=out)
        kv.mpt_kv_check()
        assert torch.equal(got, want) and torch.equal(lse, want_lse)
