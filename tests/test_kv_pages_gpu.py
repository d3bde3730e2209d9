"""The page operators: writes, merges, forks, extensions, freeing, compaction and copies, against plain
models (tests/kv_model.py), all bookkeeping and copies to the bit."""

import math
import random

import pytest

torch = pytest.importorskip("torch")

from tests import kv_model as M

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = dict(dtype=torch.int32)


@pytest.fixture(scope="module")
def kv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    B.build()
    from paper_2609_13692_gb300 import kv as K

    return K


def dev(x):
    return torch.tensor(x, **I32).cuda()


# ---------------------------------------------------------------------------
# Merge
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("parts", [1, 2, 3, 4, 5, 16])
@pytest.mark.parametrize("rows,dim", [(1, 8), (7, 96), (333, 128), (65, 1024)])
def test_merge(kv, rows, dim, parts, dtype):
    gen = torch.Generator(device="cuda").manual_seed(parts * rows + dim)
    outs = torch.randn((parts, rows, dim), generator=gen, device="cuda").to(dtype)
    lses = torch.randn((parts, rows), generator=gen, device="cuda") * 3
    empty = torch.rand((parts, rows), generator=gen, device="cuda") < 0.3
    empty[:, :1] = True  # a row without keys
    lses = torch.where(empty, -math.inf, lses)
    outs[empty] = math.nan  # no say
    out, lse = kv.mpt_kv_merge(outs, lses)
    x, z = torch.where(empty[..., None], 0.0, outs.double()), torch.logsumexp(lses.double(), 0)
    w = torch.exp(lses.double() - torch.where(torch.isinf(z), 0.0, z))
    want, most = (w[..., None] * x).sum(0), (w[..., None] * x.abs()).sum(0)
    # weights to 2^-20 (exponent of a 32-bit difference of at most 2^5), 32-bit sums, one rounding
    tol = M.UNIT[dtype] * want.abs() + (2.0 ** -19 + parts * 2.0 ** -23) * most + 2.0 ** -25
    assert bool(((out.double() - want).abs() <= tol).all())
    none = torch.isinf(z)
    assert torch.equal(torch.isneginf(lse), none) and bool((out[none] == 0).all())
    assert bool(((lse.double() - z).abs()[~none] <= 2.0 ** -20 + 2.0 ** -22 * z.abs()[~none]).all())
    again = outs.clone()
    kv.mpt_kv_merge(again, lses, out=again[0])
    assert torch.equal(again[0], out)


def test_merge_of_attention_over_parts(kv):
    """Prefix and suffix attended apart give what the whole does."""
    from tests.test_kv_attend_gpu import args, make

    c = make(1, [30], [500], 8, 2, 128, 16, BF16)
    whole, whole_lse = kv.mpt_kv_attend(*args(c))
    head = kv.mpt_kv_attend(c["q"], c["k"], c["v"], c["table"], c["at"], dev([320]), causal=False)
    tail = kv.mpt_kv_attend(c["q"], c["k"], c["v"], c["table"][:, 20:].contiguous(), c["at"], dev([180]))
    out, lse = kv.mpt_kv_merge([head[0], tail[0]], [head[1], tail[1]])
    _, _, tol, tol_lse = M.attend(*args(c), True, 1 / math.sqrt(128))
    # each part is within its own bound of its exact value, and rounded once more on the way
    assert bool(((out.double() - whole.double()).abs() <= 4 * tol).all())
    assert bool(((lse.double() - whole_lse.double()).abs() <= 4 * tol_lse).all())


def test_merge_refusals(kv):
    from paper_2609_13692_gb300.mpt import MPTError

    o, l = torch.zeros((2, 3, 16), device="cuda"), torch.zeros((2, 3), device="cuda")
    for outs, lses, st in ((torch.zeros((17, 3, 16), device="cuda"), torch.zeros((17, 3), device="cuda"), 2),
                           (torch.zeros((2, 3, 12), device="cuda"), l, 1), (torch.zeros((2, 3, 1032), device="cuda"), l, 2)):
        with pytest.raises(MPTError) as e:
            kv.mpt_kv_merge(outs, lses)
        assert e.value.status == st
    with pytest.raises(MPTError):
        kv.mpt_kv_merge(o, l, lse=l[0])
    for outs, lses in (([], []), (o, l[:1]), (o.double(), l), (o, l.half()), (o, l[:, :2]), ([o[0], o[1, :2]], l)):
        with pytest.raises(ValueError):
            kv.mpt_kv_merge(outs, lses)
    out, lse = kv.mpt_kv_merge(o[:, :0], l[:, :0])
    assert out.shape == (0, 16) and lse.shape == (0,)


# ---------------------------------------------------------------------------
# Write
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("kv_heads,dim,page,dtype", [(2, 64, 16, BF16), (1, 8, 8, F16), (3, 72, 32, BF16), (8, 256, 256, F16)])
def test_write(kv, kv_heads, dim, page, dtype, order):
    rng = random.Random(dim)
    q_lens = [1, 0, 5, 300, 0, 1, 33] + [rng.randint(0, 2) for _ in range(60)]
    kv_lens = [n + rng.randint(0, 400) for n in q_lens]
    kv_lens[2] = 3  # two tokens stand before the beginning
    width = max(-(-n // page) for n in kv_lens)
    ids = list(range(len(q_lens) * width + 3))
    rng.shuffle(ids)
    n_pages = len(ids)
    table = torch.tensor(ids[:len(q_lens) * width], **I32).view(len(q_lens), width)
    table[3, 1] = -1
    table[6, 0] = n_pages
    shape = (n_pages, 2, page, kv_heads, dim) if order == "token" else (n_pages, 2, kv_heads, page, dim)
    pool = torch.randn(shape, device="cuda").to(dtype)
    k, v = (pool[:, 0], pool[:, 1]) if order == "token" else (pool[:, 0].transpose(1, 2), pool[:, 1].transpose(1, 2))
    at = [0]
    for n in q_lens:
        at.append(at[-1] + n)
    extra = 2  # tokens past the last request's are nobody's
    wide = torch.randn((at[-1] + extra, 2 * kv_heads + 1, dim + 8), device="cuda").to(dtype)
    k_new, v_new = wide[:, :kv_heads, :dim], wide[:, kv_heads + 1:, 8:]
    want_k, want_v = k.clone(), v.clone()
    for i, n in enumerate(q_lens):
        for t in range(n):
            pos = kv_lens[i] - n + t
            p = int(table[i, pos // page]) if pos >= 0 else -1
            if 0 <= p < n_pages:
                want_k[p, pos % page], want_v[p, pos % page] = k_new[at[i] + t], v_new[at[i] + t]
    kv.mpt_kv_write(k_new, v_new, k, v, table.cuda(), dev(at), dev(kv_lens))
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


def test_write_refusals(kv):
    from paper_2609_13692_gb300.mpt import MPTError

    pool = torch.zeros((4, 2, 16, 2, 64), dtype=BF16, device="cuda")
    k, v, table, at, lens = pool[:, 0], pool[:, 1], dev([[0, 1]]), dev([0, 1]), dev([5])
    new = torch.zeros((1, 2, 64), dtype=BF16, device="cuda")
    kv.mpt_kv_write(new, new, k, v, table, at, lens)
    kv.mpt_kv_write(new[:0], new[:0], k, v, table, dev([0, 0]), lens)
    for a, b in ((new.float(), new), (new[:, :1], new), (new, torch.cat([new, new]))):
        with pytest.raises(ValueError):
            kv.mpt_kv_write(a, b, k, v, table, at, lens)
    with pytest.raises(MPTError) as e:
        odd = torch.zeros((1, 2, 72), dtype=BF16, device="cuda")[:, :, 1:65]
        kv.mpt_kv_write(odd, odd, k, v, table, at, lens)
    assert e.value.status == 1


# ---------------------------------------------------------------------------
# Bookkeeping
# ---------------------------------------------------------------------------

def same(book, tensors):
    want = book.tensors("cpu")
    return all(torch.equal(a, b.cpu()) for a, b in zip(want, tensors))


@pytest.mark.parametrize("rows,width,n_pages,page,stride", [(40, 9, 400, 8, 9), (300, 33, 4001, 16, 50), (7, 2, 31, 256, 2),
                                                           (64, 1, 64, 16, 3), (1500, 6, 20_000, 32, 6)])
def test_bookkeeping(kv, rows, width, n_pages, page, stride):
    """Random steps of all four calls follow the host's bookkeeping exactly."""
    rng = random.Random(rows)
    book = M.Book(rows, width, n_pages, page)
    t = book.tensors("cuda", stride)
    for step in range(24):
        full = [r for r in range(rows) if book.lens[r] > 0]
        empty = [r for r in range(rows) if book.lens[r] == 0]
        rng.shuffle(full)
        rng.shuffle(empty)
        kind = step % 4
        if kind == 0:  # grow
            left, pick, more = len(book.free_ids()), [], []
            for r in rng.sample(range(rows), rows // 2):
                n = rng.randint(0, min(3 * page, width * page - book.lens[r]))
                need = -(-(book.lens[r] + n) // page) - -(-book.lens[r] // page)
                if need <= left:
                    left -= need
                    pick.append(r)
                    more.append(n)
            book.extend(pick, more)
            status = kv.mpt_kv_extend(*t, page, dev(pick), dev(more))
        elif kind == 1 and full:  # fork
            dst = empty[:min(len(empty), len(book.free_ids()), rows // 3)]
            src = [rng.choice(full) for _ in dst]
            keep = [rng.choice([0, book.lens[s], rng.randint(0, book.lens[s])]) for s in src]
            pairs = book.fork(src, dst, keep)
            old, fresh, status = kv.mpt_kv_fork(*t, page, dev(src), dev(dst), dev(keep))
            assert list(zip(old.tolist(), fresh.tolist())) == pairs
        elif kind == 2:
            gone = full[:len(full) // 3] + empty[:2]
            book.free(gone)
            status = kv.mpt_kv_free(*t, page, dev(gone))
        else:
            moves = book.compact()
            old, fresh, status = kv.mpt_kv_compact(*t, page)
            assert old.shape[0] == n_pages // 2
            assert list(zip(old.tolist(), fresh.tolist())) == moves + [(-1, -1)] * (n_pages // 2 - len(moves))
        assert status.tolist() == [0, len(book.free_ids())]
        assert same(book, t), (step, kind)


def test_bookkeeping_of_long_lists(kv):
    """As many entries as a call takes, in a table of many rows."""
    rows, page, n = 100_000, 8, 16_384
    t = (torch.full((rows, 2), -1, **I32).cuda(), torch.zeros(rows, **I32).cuda(), torch.zeros(60_000, **I32).cuda())
    pick = torch.randperm(rows)[:2 * n].to(torch.int32)
    first, second = pick[:n].cuda(), pick[n:].cuda()
    more = torch.randint(0, 16, (n,)).to(torch.int32)
    assert kv.mpt_kv_extend(*t, page, first, more.cuda()).tolist()[0] == 0
    need = -(-more // page)
    at = need.cumsum(0) - need
    for i in range(2):  # pages in list order, the lowest first
        want = torch.where(need > i, at + i, -1).to(torch.int32)
        assert torch.equal(t[0][first.long(), i].cpu(), want)
    keep = torch.minimum(more, torch.randint(0, 16, (n,)).to(torch.int32))
    old, fresh, status = kv.mpt_kv_fork(*t, page, first, second, keep.cuda())
    part = keep % page > 0
    used = int(need.sum())
    assert status.tolist() == [0, 60_000 - used - int(part.sum())]
    rank = part.cumsum(0) - 1
    assert torch.equal(fresh.cpu(), torch.where(part, used + rank, -1).to(torch.int32))
    assert torch.equal(old.cpu(), torch.where(part, at + keep // page, -1).to(torch.int32))
    assert torch.equal(t[1][second.long()].cpu(), keep)
    refs = torch.zeros(60_000, **I32)
    refs[:used + int(part.sum())] = 1
    full = keep // page
    refs[at[full > 0]] += 1
    assert torch.equal(t[2].cpu(), refs)
    assert kv.mpt_kv_free(*t, page, first).tolist()[0] == 0
    assert kv.mpt_kv_free(*t, page, second).tolist() == [0, 60_000]


def test_bookkeeping_of_holes(kv):
    """Entries that the cache does not hold stay holes and hold no reference."""
    book = M.Book(4, 4, 20, 8)
    book.extend([0], [27])
    book.table[0][1] = -1
    book.refs[1] = 0
    t = book.tensors("cuda")
    pairs = book.fork([0, 0], [1, 2], [27, 12])
    old, fresh, status = kv.mpt_kv_fork(*t, 8, dev([0, 0]), dev([1, 2]), dev([27, 12]))
    assert list(zip(old.tolist(), fresh.tolist())) == pairs and pairs[1] == (-1, -1)
    # a part page that is a hole is one in the copy as well
    assert same(book, t)
    book.free([0, 1])
    kv.mpt_kv_free(*t, 8, dev([0, 1]))
    assert same(book, t)


def test_bookkeeping_refused_on_the_device(kv):
    """A call that cannot be done changes nothing and says why."""
    page = 16
    book = M.Book(8, 4, 10, page)
    book.extend([0, 1, 2], [60, 17, 1])
    t = book.tensors("cuda")
    before = [x.clone() for x in t]
    free = len(book.free_ids())
    assert free == 3
    cases = [
        (kv.mpt_kv_extend, ([0, 8], [1, 1]), 1), (kv.mpt_kv_extend, ([0, -1], [1, 1]), 1),
        (kv.mpt_kv_extend, ([2, 2], [1, 1]), 1), (kv.mpt_kv_extend, ([2], [-1]), 1), (kv.mpt_kv_extend, ([0], [5]), 4),
        (kv.mpt_kv_extend, ([3], [2 ** 31 - 1]), 4), (kv.mpt_kv_extend, ([3, 4], [33, 16]), 2),
        (kv.mpt_kv_fork, ([0, 1], [3, 3], [16, 16]), 1), (kv.mpt_kv_fork, ([0], [1], [16]), 1),
        (kv.mpt_kv_fork, ([0], [3], [61]), 1), (kv.mpt_kv_fork, ([0], [3], [-1]), 1), (kv.mpt_kv_fork, ([8], [3], [0]), 1),
        (kv.mpt_kv_fork, ([0], [-2], [0]), 1), (kv.mpt_kv_fork, ([0, 0, 0, 0], [3, 4, 5, 6], [1, 1, 1, 1]), 2),
        (kv.mpt_kv_free, ([0, 0],), 1), (kv.mpt_kv_free, ([0, 99],), 1),
    ]
    for call, lists, flag in cases:
        got = call(*t, page, *[dev(x) for x in lists])
        status = got[-1] if isinstance(got, tuple) else got
        assert status.tolist() == [flag, free], (call.__name__, lists)
        if call is kv.mpt_kv_fork:
            assert bool((got[0] == -1).all()) and bool((got[1] == -1).all())
        assert all(torch.equal(a, b) for a, b in zip(before, t)), (call.__name__, lists)
    status = kv.mpt_kv_extend(*t, page, dev([3, 4]), dev([32, 16]))  # the last pages
    assert status.tolist() == [0, 0]
    status = kv.mpt_kv_extend(*t, page, dev([]), dev([]))
    assert status.tolist() == [0, 0]


def test_bookkeeping_refusals(kv):
    from paper_2609_13692_gb300.mpt import MPTError

    t = M.Book(4, 4, 10, 16).tensors("cuda")
    wide = (torch.full((20_000, 1), -1, **I32).cuda(), torch.zeros(20_000, **I32).cuda(), t[2])
    for call, st in ((lambda: kv.mpt_kv_free(*t, 12, dev([0])), 1), (lambda: kv.mpt_kv_free(*t, 16, dev([0, 1, 2, 3, 0])), 2),
                     (lambda: kv.mpt_kv_free(*wide, 16, torch.arange(16_385, **I32).cuda()), 2)):
        with pytest.raises(MPTError) as e:
            call()
        assert e.value.status == st
    for call in (lambda: kv.mpt_kv_free(t[0].long(), t[1], t[2], 16, dev([0])), lambda: kv.mpt_kv_free(t[0], t[1][:2], t[2], 16, dev([0])),
                 lambda: kv.mpt_kv_extend(*t, 16, dev([0]), dev([1, 2])), lambda: kv.mpt_kv_free(*t, 16, torch.zeros(1, **I32))):
        with pytest.raises(ValueError):
            call()


# ---------------------------------------------------------------------------
# Copies
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("planes,n_pages,shape,dtype", [(1, 9, (8,), BF16), (3, 200, (2, 16, 2, 64), BF16), (2, 50, (33, 8), F32),
                                                        (5, 12, (2, 256, 8, 128), F16), (64, 700, (16, 3, 24), BF16)])
def test_copy_pages(kv, planes, n_pages, shape, dtype):
    rng = random.Random(n_pages)
    pool = torch.randn((planes + 1, n_pages, *shape), device="cuda").to(dtype)[:planes]
    want = pool.clone()
    ids = rng.sample(range(n_pages), n_pages)
    dst, src = ids[:n_pages // 3], [rng.choice(ids[n_pages // 3:]) for _ in range(n_pages // 3)]
    for s, d in zip(src, dst):
        want[:, d] = want[:, s]
    for bad in (-1, n_pages, -2 ** 31):
        at = rng.randint(0, len(src))
        src.insert(at, bad)
        dst.insert(at, ids[-1])
        dst.append(bad)
        src.append(ids[-1])
    kv.mpt_kv_copy_pages(pool, dev(src), dev(dst))
    assert torch.equal(pool, want)
    kv.mpt_kv_copy_pages(pool, dev([]), dev([]))


def test_copy_pages_beyond_32_bits(kv):
    pool = torch.empty((3, 50_000, 65_536), dtype=torch.uint8, device="cuda")  # 9.8 GB
    for p in range(3):
        pool[p, 7].random_(0, 255)
    kv.mpt_kv_copy_pages(pool, dev([7]), dev([49_999]))
    assert torch.equal(pool[:, 49_999], pool[:, 7])


def test_copy_pages_refusals(kv):
    from paper_2609_13692_gb300.mpt import MPTError

    pool = torch.zeros((2, 4, 10), dtype=BF16, device="cuda")  # pages of 20 bytes
    with pytest.raises(MPTError) as e:
        kv.mpt_kv_copy_pages(pool, dev([0]), dev([1]))
    assert e.value.status == 1
    pool = torch.zeros((2, 4, 16, 8), dtype=BF16, device="cuda")
    for a, b, c in ((pool[:, :, :, :4], dev([0]), dev([1])), (pool[0, 0], dev([0]), dev([1])), (pool, dev([0]), dev([1, 2])),
                    (pool[:0], dev([0]), dev([1])), (pool, torch.zeros(1, **I32), dev([1]))):
        with pytest.raises(ValueError):
            kv.mpt_kv_copy_pages(a, b, c)
