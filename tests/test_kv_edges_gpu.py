"""The paged-cache operators at the edges of their ranges, against the models of tests/kv_model.py."""

import math
import random

import pytest

torch = pytest.importorskip("torch")

from tests import kv_model as M
from tests.test_kv_attend_gpu import BF16, F16, args, check, kv, make  # noqa: F401 (kv: the fixture)

pytestmark = pytest.mark.gpu


def bits(x):
    return x.view(torch.int32 if x.dtype is torch.float32 else torch.int16)


@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(8, 2, 128, BF16), (8, 2, 64, F16), (4, 4, 96, BF16), (6, 1, 200, BF16)])
def test_noted_values_beside_items_of_one_row_tile(kv, heads, kv_heads, dim, dtype):  # noqa: F811
    """Requests of two row tiles whose new values are not finite, each before several of one row tile: the rows
    that add such keys one by one are still at it while the others go on, and keep their own notes."""
    toks = 128 // (heads // kv_heads)
    q_lens, kv_lens = [], []
    for i in range(120):
        q_lens += [toks + 1 + i % toks, 1, 1, 3, 1, 2, 1]
        kv_lens += [toks + 9 + i % toks + i % 50, 1 + i % 40, 7, 3, 30, 2 + i % 9, 1]
    c = make(31, q_lens, kv_lens, heads, kv_heads, dim, 16, dtype)
    for i in range(0, len(q_lens), 7):
        keys = torch.arange(kv_lens[i] - q_lens[i] + 1, kv_lens[i], 2 if i % 2 else 3, device="cuda")
        pages = c["table"][i].long()[keys // 16]
        c["v"][pages, keys % 16, :, 5] = math.inf
        c["v"][pages[-1], keys[-1] % 16, :, 33] = math.nan
    want, want_lse, tol, tol_lse = M.attend(*args(c), True, 1 / math.sqrt(dim))
    out, lse = kv.mpt_kv_attend(*args(c), max_q_len=2 * toks)
    kv.mpt_kv_check()
    assert bool(((lse.double() - want_lse).abs() <= tol_lse).all())
    finite = torch.isfinite(want)
    assert bool(((out.double() - want).abs()[finite] <= tol[finite]).all())
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.isposinf(out), torch.isposinf(want))
    for _ in range(5):
        again = kv.mpt_kv_attend(*args(c), max_q_len=2 * toks)
        assert torch.equal(bits(again[0]), bits(out)) and torch.equal(bits(again[1]), bits(lse))


@pytest.mark.parametrize("hint", [0, 1])
def test_offsets_that_decrease_do_nothing(kv, hint):  # noqa: F811
    """Offsets that give every second of 8,192 requests the same 2^17 tokens, 2^31 items in all."""
    batch, tokens, heads, kv_heads, dim = 8192, 1 << 17, 1024, 8, 8
    assert batch // 2 * (tokens // (2 * (128 // (heads // kv_heads)))) * kv_heads == 1 << 31
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((2, 8, kv_heads, dim), dtype=BF16, device="cuda")
    at = torch.zeros(batch + 1, **i32)
    at[1::2] = tokens
    q = torch.zeros((tokens, heads, dim), dtype=BF16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((tokens, heads), 7.0, device="cuda")
    kv.mpt_kv_attend(q, pool, pool, torch.zeros((batch, 1), **i32), at, torch.full((batch,), 8, **i32), max_q_len=hint, out=out,
                     lse=lse)
    kv.mpt_kv_check()
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
    # one step back among few requests
    c = make(32, [3, 4, 60], [30, 40, 70], 4, 2, 64, 16, BF16)
    c["at"][2] = 2
    out = torch.full_like(c["q"], 7.0)
    kv.mpt_kv_attend(*args(c), max_q_len=hint, out=out)
    kv.mpt_kv_check()
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page,dim,q_len,rest", [(32, 64, 1, 32), (32, 128, 40, 27), (16, 128, 2, 16), (8, 256, 50, 5)])
def test_keys_up_to_the_last_of_32_bits(kv, page, dim, q_len, rest, causal):  # noqa: F811
    """A sparse table as wide as it may be, its last page beside 2^31; the keys that are there, as a cache of their own."""
    width = (2 ** 31 - 1) // page
    gen = torch.Generator(device="cuda").manual_seed(page)
    pool = torch.randn((2, 7, page, 2, dim), generator=gen, device="cuda").to(BF16)
    pool[:, 5, rest:] = math.nan  # beyond the last key
    i32 = dict(dtype=torch.int32, device="cuda")
    near = -(-q_len // page) + 1  # the pages of the new tokens, one more
    table = torch.full((1, width), -1, **i32)
    there = [0, 12_345_678 // page, *range(width - near, width)]
    pages = [3, 6, *([1, 0, 2, 4, 1, 0, 2] * 2)[:near - 1], 5]
    table[0, torch.tensor(there, device="cuda")] = torch.tensor(pages, **i32)
    q = torch.randn((q_len, 4, dim), generator=gen, device="cuda").to(BF16)
    at = torch.tensor([0, q_len], **i32)
    lens = (width - 1) * page + rest
    assert lens > 2 ** 31 - 64
    out, lse = kv.mpt_kv_attend(q, pool[0], pool[1], table, at, torch.tensor([lens], **i32), causal=causal, max_q_len=q_len)
    kv.mpt_kv_check()
    want, want_lse, tol, tol_lse = M.attend(q, pool[0], pool[1], torch.tensor([pages], **i32), at,
                                            torch.tensor([(len(pages) - 1) * page + rest], **i32), causal, 1 / math.sqrt(dim))
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - want_lse).abs() <= tol_lse).all())


@pytest.mark.parametrize("q_len,group", [(1, 4), (40, 2), (40, 1)])
@pytest.mark.parametrize("dtype,dim", [(F16, 64), (F16, 128), (F16, 256), (BF16, 128)])
def test_many_keys_of_small_weight(kv, dtype, dim, q_len, group):  # noqa: F811
    """The first 128 keys outweigh each of the other 131,072 by 2^25 and more; together those are a part of the
    output.  So many requests that most are some block's alone."""
    n, page, batch = 131_200, 64, 1000 if q_len == 1 else 400
    i32 = dict(dtype=torch.int32, device="cuda")
    for weight in (2.9e-8, 2.0 ** -26, 1e-9):
        pool = torch.zeros((2, n // page + 1, page, 1, dim), dtype=dtype, device="cuda")
        k, v = pool
        q = torch.zeros((batch * q_len, group, dim), dtype=dtype, device="cuda")
        q[..., 0] = 4.0
        # scores are 4 times the key's first element at scale 1: 0 for the far keys, -ln(weight) for the first
        k[:2, :, 0, 0] = -math.log(weight) / 4
        v.normal_(generator=torch.Generator(device="cuda").manual_seed(dim))
        v += 1.0
        v[:2] = 0
        c = (q, k, v, torch.arange(n // page, **i32).repeat(batch, 1), torch.arange(0, batch * q_len + 1, q_len, **i32),
             torch.full((batch,), n, **i32))
        out, lse = kv.mpt_kv_attend(*c, causal=False, scale=1.0, max_q_len=q_len)
        kv.mpt_kv_check()
        s = torch.zeros(n, dtype=torch.float64, device="cuda")
        s[:128] = 4 * float(k[0, 0, 0, 0])
        z = torch.logsumexp(s, 0)
        p, x = torch.exp(s - z), v.view(-1, dim)[:n].double()
        want = p @ x
        # each probability rounded once, relatively or (f16) by 2^-25 of 2^11 times its value; the sums' and
        # exponentials' errors as in tests/kv_model.py; the result rounded, relatively or by half the least f16
        u, err = M.UNIT[dtype], 2.0 ** -20 + n * 2.0 ** -24
        tol = u * want.abs() + (u + 2 * err) * (1 + u) * (p @ x.abs()) + 2.0 ** -25
        if dtype is F16:
            tol = tol + 2.0 ** -36 * p[0] * x.abs().sum(0)
        assert bool(((out.double() - want).abs() <= tol).all()), weight
        assert float((lse.double() - z).abs().max()) <= err + 2.0 ** -20 + 2.0 ** -21 * float(z)


def test_gradients_are_refused(kv):  # noqa: F811
    """There is no backward pass: tensors that require gradients are taken only where none are recorded."""
    c = make(33, [1, 40], [30, 70], 4, 2, 64, 16, BF16)
    out, lse = kv.mpt_kv_attend(*args(c))
    parts, sums = torch.stack([out, out]), torch.stack([lse, lse])
    want = kv.mpt_kv_merge(parts, sums)
    new = c["k"][0, :1].clone()
    one = (c["table"][:1], torch.tensor([0, 1], dtype=torch.int32, device="cuda"), c["lens"][:1])
    pages = torch.zeros((1, 4, 16, 2, 64), dtype=BF16, device="cuda")
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")

    def req(t):
        return t.detach().clone().requires_grad_()

    calls = [lambda: kv.mpt_kv_attend(*args(dict(c, q=req(c["q"])))), lambda: kv.mpt_kv_attend(*args(dict(c, k=req(c["k"])))),
             lambda: kv.mpt_kv_attend(*args(dict(c, v=req(c["v"])))), lambda: kv.mpt_kv_attend(*args(c), out=req(out)),
             lambda: kv.mpt_kv_attend(*args(c), lse=req(lse)), lambda: kv.mpt_kv_merge(req(parts), sums),
             lambda: kv.mpt_kv_merge(parts, req(sums)), lambda: kv.mpt_kv_merge([out, req(out)], [lse, lse]),
             lambda: kv.mpt_kv_merge(iter([out, out]), iter([req(lse), lse])), lambda: kv.mpt_kv_merge(parts, sums, out=req(out)),
             lambda: kv.mpt_kv_write(req(new), new, c["k"], c["v"], *one), lambda: kv.mpt_kv_write(new, req(new), c["k"], c["v"], *one),
             lambda: kv.mpt_kv_copy_pages(req(pages), ids, ids)]
    for call in calls:
        with pytest.raises(ValueError, match="no backward"):
            call()
    with torch.no_grad():
        got = kv.mpt_kv_attend(*args(dict(c, q=req(c["q"]))))
        assert torch.equal(got[0], out) and not got[0].requires_grad
        assert torch.equal(kv.mpt_kv_merge(req(parts), sums)[0], want[0])
    with torch.inference_mode():
        assert torch.equal(kv.mpt_kv_attend(*args(c))[0], out)


@pytest.mark.parametrize("heads,kv_heads,dim", [(82, 2, 64), (43, 1, 256), (65, 1, 128), (200, 2, 96), (128, 1, 128), (128, 1, 200)])
def test_large_groups(kv, heads, kv_heads, dim):  # noqa: F811
    """41 to 128 query heads of a KV head: row tiles of three, two and one whole tokens."""
    for causal in (True, False):
        check(kv, make(34, [1, 1, 0, 1], [300, 1, 5, 130], heads, kv_heads, dim, 16, BF16, poison=True), causal, hint=1)
        check(kv, make(35, [1, 7, 2, 30], [64, 7, 1, 257], heads, kv_heads, dim, 32, F16, holes=0.2, poison=True), causal, hint=30)


def test_chunks_of_more_requests_than_the_large_kernel_lists(kv):  # noqa: F811
    """Above 8,192 requests the small kernel takes chunks too."""
    rng = random.Random(36)
    q_lens = [rng.choice([1, 3, 17, 70]) if i % 41 == 0 else 0 for i in range(8_200)]
    kv_lens = [max(0, n + rng.choice([-2, 0, 9, 150])) if n else i % 2 for i, n in enumerate(q_lens)]
    for dim, dtype in ((64, BF16), (256, F16)):
        check(kv, make(36, q_lens, kv_lens, 4, 2, dim, 16, dtype, poison=True), hint=70)


def test_calls_on_two_streams_at_once(kv):  # noqa: F811
    """Two streams in turn and together, each with outputs and a workspace of its own."""
    cases = [make(37, [1] * 20, [3_000] * 20, 8, 2, 128, 16, BF16), make(38, [300, 1, 40], [4_000, 900, 333], 8, 2, 128, 16, BF16),
             make(39, [1, 1], [60_000, 5], 4, 4, 64, 64, F16), make(40, [90], [9_000], 4, 2, 256, 16, F16)]
    hints = [1, 300, 1, 90]
    want = [kv.mpt_kv_attend(*args(c), max_q_len=h) for c, h in zip(cases, hints)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for first, second in ((0, 1), (1, 2), (3, 1), (1, 1), (0, 0)):
        mine = []
        for i in (first, second):
            c = cases[i]
            ws = torch.empty(kv.mpt_kv_attend_workspace_bytes(c["q"].shape[2]), dtype=torch.uint8, device="cuda")
            mine.append((i, [(torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")) for _ in range(8)], ws))
        torch.cuda.synchronize()
        for n in range(8):
            for s, (i, outs, ws) in zip(streams, mine):
                kv.mpt_kv_attend(*args(cases[i]), max_q_len=hints[i], out=outs[n][0], lse=outs[n][1], workspace=ws, stream=s.cuda_stream)
        torch.cuda.synchronize()
        kv.mpt_kv_check()
        for i, outs, _ in mine:
            for out, lse in outs:
                assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]), (first, second, i)


@pytest.mark.parametrize("q_len,dim", [(1, 128), (1, 256), (50, 64), (50, 256)])
def test_heads_before_tokens(kv, q_len, dim):  # noqa: F811
    """q and out stored head by head: the heads' stride is the larger one."""
    c = make(41, [q_len, 1, q_len], [77, 500, 250], 6, 2, dim, 16, BF16, "head")
    c["q"] = c["q"].transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty((6, c["q"].shape[0], dim), dtype=BF16, device="cuda").transpose(0, 1)
    check(kv, c, hint=q_len, out=out)


def test_writes_by_offsets_that_decrease(kv):  # noqa: F811
    """Tokens that the offsets give to no request, as they are looked up, are dropped."""
    at = [4, 6, 2, 3]
    batch, tokens, page = 3, 8, 8
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((2, 9, page, 1, 8), dtype=BF16, device="cuda")
    new = torch.ones((tokens, 1, 8), dtype=BF16, device="cuda")
    kv.mpt_kv_write(new, new, pool[0], pool[1], torch.arange(9, **i32).view(3, 3), torch.tensor(at, **i32),
                    torch.full((batch,), 20, **i32))
    kv.mpt_kv_check()
    for side in pool:
        written = side[:, :, 0, 0].reshape(batch, 3 * page).nonzero().tolist()
        allowed = {(i, 20 - (at[i + 1] - at[i]) + t - at[i]) for i in range(batch) for t in range(max(at[i], 0), min(at[i + 1], tokens))}
        assert {tuple(x) for x in written} <= allowed
