"""Results of the turned writes and of reading codes back that share memory with one another or with what the
call reads are refused, parts of one tensor that interleave are not: the rule (csrc/kv_overlap.h) compiled
for the host, against the bytes themselves; the calls' refusals, for which no GPU is needed; and calls on
parts of one tensor."""

import ctypes
import itertools
import os
import random
import struct
import subprocess

import pytest

from paper_2609_13692_gb300 import build as B

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "%s/paper_2609_13692_gb300/csrc/kv_overlap.h"
extern "C" int overlap(const mpt::HeadRuns* a, const mpt::HeadRuns* b) { return mpt::heads_overlap(*a, *b); }
"""
DIM = 64


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    at = tmp_path_factory.mktemp("overlap")
    (at / "o.cpp").write_text(SOURCE % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(at / "o.so"), str(at / "o.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "o.so"))
    lib.overlap.argtypes = [ctypes.c_char_p] * 2

    def call(a, b):
        one, two = (bool(lib.overlap(struct.pack("@6q", *x), struct.pack("@6q", *y))) for x, y in ((a, b), (b, a)))
        assert one == two
        return one

    return call


def runs(at, s, tokens, heads, size=2, dim=DIM):
    return at, dim * size, tokens, heads, s[0] * size, s[1] * size


def touched(r):
    at, run, tokens, heads, s0, s1 = r
    return {at + t * s0 + h * s1 + e for t in range(tokens) for h in range(heads) for e in range(0, run, 16)}


LAYOUTS = [  # strides of tokens and heads
    lambda h, t: (h * DIM, DIM), lambda h, t: (DIM, t * DIM), lambda h, t: (2 * h * DIM, DIM), lambda h, t: (2 * h * DIM, 2 * DIM),
    lambda h, t: ((h + 3) * DIM + 8, DIM), lambda h, t: (DIM + 8, (t + 1) * (DIM + 8)), lambda h, t: (8, 16),
]


@pytest.mark.parametrize("size", [2, 4])
def test_rule(overlap, size):
    """Every pair of layouts at many distances, against the bytes."""
    rng = random.Random(size)
    found = {True: 0, False: 0}
    for one, two in itertools.product(LAYOUTS, repeat=2):
        for _ in range(200):
            tokens, heads, more = rng.choice([1, 2, 3, 7]), rng.choice([1, 2, 4]), rng.choice([1, 2, 4])
            d = rng.choice([0, 16, DIM * size, -DIM * size, heads * DIM * size, 16 * rng.randint(-400, 400)])
            a, b = runs(1 << 40, one(heads, tokens), tokens, heads, size), runs((1 << 40) + d, two(more, tokens), tokens, more, size)
            got = overlap(a, b)
            assert got == bool(touched(a) & touched(b)), (a, b)
            found[got] += 1
    assert min(found.values()) > 1000


def test_rule_at_the_largest_sizes(overlap):
    """2^31 - 1 tokens, strides of 2^40 bytes: no product overflows, and ordinary layouts are found out at once."""
    n, far = 2 ** 31 - 1, ((1 << 38) - 8, DIM)
    assert overlap(runs(1 << 40, far, n, 1, 4), runs(1 << 40, far, n, 1, 4))
    assert not overlap(runs(1 << 40, far, n, 1, 4), runs((1 << 40) + 256, far, n, 1, 4))
    row = (1024 * DIM, DIM)
    assert overlap(runs(1 << 40, row, n, 1024), runs((1 << 40) + 1024 * DIM * 2 * (n - 1), row, n, 1024))
    assert not overlap(runs(1 << 40, row, n, 1024), runs((1 << 40) + 1024 * DIM * 2 * n, row, n, 1024))
    packed = (48 * 128, 128)  # queries, keys and values of one tensor
    parts = [runs(1 << 40, packed, n, 32, 2, 128), runs((1 << 40) + 32 * 256, packed, n, 8, 2, 128), runs((1 << 40) + 40 * 256, packed, n, 8, 2, 128)]
    assert not any(overlap(a, b) for a, b in itertools.combinations(parts, 2))
    assert overlap(parts[0], runs((1 << 40) + 31 * 256, packed, n, 8, 2, 128))
    swapped = (128, n * 128)  # heads before tokens
    assert not overlap(runs(1 << 40, swapped, n, 8, 2, 128), runs((1 << 40) + 8 * n * 256, swapped, n, 8, 2, 128))
    assert overlap(runs(1 << 40, swapped, n, 8, 2, 128), runs((1 << 40) + 8 * n * 256 - 256, swapped, n, 8, 2, 128))


A, FAR = 1 << 40, 1 << 44  # addresses that nothing reads: every call below returns before it would


@pytest.fixture(scope="module")
def lib():
    B.build()
    from paper_2609_13692_gb300 import mpt as M

    return M.load()


def cache4(heads, batch=2):
    from paper_2609_13692_gb300 import kv

    return kv._CACHE4.pack(FAR, 1152 * heads, 1152, 10, 16, heads, DIM, batch, FAR, 5, 5, FAR, FAR)


def cache(heads, batch=2):
    from paper_2609_13692_gb300 import kv

    return kv._CACHE.pack(FAR, FAR, 16 * heads * DIM, heads * DIM, DIM, 16 * heads * DIM, heads * DIM, DIM, 0, 10, 16, heads, DIM, batch, FAR, 5, 5, FAR, FAR)


def pair(s):
    return struct.pack("@2q", *s)


def read(lib, k, v, s=(2 * DIM, DIM), type=0, batch=2):
    return lib.mpt_kv4_read(cache4(2, batch), type, k, pair(s), v, pair(s), 5, 0)


def write(lib, codes, q, q_out, qs=(256, DIM), os=(256, DIM), k=FAR, v=FAR, s=(2 * DIM, DIM), batch=2):
    from paper_2609_13692_gb300 import kv

    turn = kv._TURN.pack(FAR, DIM, 100, DIM, 0, 4, 0, q, q_out, *qs, *os)
    if codes:
        return lib.mpt_kv4_write(cache4(2, batch), turn, 0, k, pair(s), v, pair(s), 5, 0)
    return lib.mpt_kv_write_rotated(cache(2, batch), turn, k, pair(s), v, pair(s), 5, 0)


def test_reads_are_refused(lib):
    for d in (0, 16, 128, -128, 5 * 256 - 16, -5 * 256 + 16):
        assert read(lib, A, A + d) == 1, d
    assert read(lib, A, A + 5 * 256, type=2) == 1  # 32 bits: twice as long
    assert read(lib, A, A + 256, s=(256, 128)) == 1  # every second head
    assert read(lib, A, A, batch=0) == 0  # nothing is written


@pytest.mark.parametrize("codes", [True, False])
def test_writes_are_refused(lib, codes):
    for qs, os, d in [((256, 64), (256, 64), 16), ((256, 64), (256, 64), 128), ((256, 64), (256, 64), 1024), ((512, 64), (512, 64), 384),
                      ((512, 64), (256, 64), 512), ((64, 320), (64, 320), 128), ((256, 64), (256, 64), -5 * 512 + 16)]:
        assert write(lib, codes, A, A + d, qs, os) == 1, (qs, os, d)
    s = (8 * DIM, DIM)  # packed: queries, two heads of keys, two of values
    packed = dict(k=A + 4 * 128, v=A + 6 * 128, s=s, qs=s, os=s)
    for d in (16, 128, 3 * 128, 6 * 128, 8 * 128 + 4 * 128):
        assert write(lib, codes, FAR, A + d, **packed) == 1, d
    assert write(lib, codes, A, A + 16, batch=0) == 0


@pytest.mark.gpu
def test_parts_of_one_tensor():
    """Queries turned in place in a packed tensor of queries, keys and values, and keys and values read back
    into one tensor: as into tensors of their own."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    B.build()
    from paper_2609_13692_gb300 import kv
    from tests import kv4_model as K

    gen = torch.Generator(device="cuda").manual_seed(3)
    n, heads, kv_heads = 37, 4, 2
    i32 = dict(dtype=torch.int32, device="cuda")
    where = torch.tensor([[2, 0, 4]], **i32), torch.tensor([0, n], **i32), torch.tensor([41], **i32)
    turns = torch.from_numpy(K.angles(41, DIM)).cuda()
    qkv = torch.randn((n, heads + 2 * kv_heads, DIM), generator=gen, device="cuda").bfloat16()
    q, k, v = (x.clone() for x in qkv.split([heads, kv_heads, kv_heads], 1))
    pages = torch.zeros((5, kv_heads, kv.mpt_kv4_page_bytes(16, DIM)), dtype=torch.uint8, device="cuda")
    pool = torch.zeros((2, 5, 16, kv_heads, DIM), dtype=torch.bfloat16, device="cuda")
    same, same_pool, packed = pages.clone(), pool.clone(), [qkv.clone(), qkv.clone()]
    want = kv.mpt_kv4_write(k, v, pages, *where, rotation=turns, q=q)
    kv.mpt_kv_write_rotated(k, v, turns, pool[0], pool[1], *where)
    pq, pk, pv = packed[0].split([heads, kv_heads, kv_heads], 1)
    assert torch.equal(kv.mpt_kv4_write(pk, pv, same, *where, rotation=turns, q=pq, q_out=pq), want) and torch.equal(same, pages)
    pq, pk, pv = packed[1].split([heads, kv_heads, kv_heads], 1)
    kv.mpt_kv_write_rotated(pk, pv, turns, same_pool[0], same_pool[1], *where, q=pq, q_out=pq)
    assert torch.equal(pq, want) and torch.equal(same_pool, pool) and torch.equal(packed[0], packed[1])
    wide = torch.randn((n, 2 * heads, DIM), generator=gen, device="cuda").bfloat16()
    wide[:, :heads] = q
    assert torch.equal(kv.mpt_kv4_write(k, v, same, *where, rotation=turns, q=wide[:, :heads], q_out=wide[:, heads:]), want)
    for dtype in (torch.bfloat16, torch.float32):
        k_want, v_want = kv.mpt_kv4_read(pages, *where, n, DIM, dtype=dtype)
        for shape, part in (((n, 2, kv_heads, DIM), lambda t, i: t[:, i]), ((n, kv_heads, 2, DIM), lambda t, i: t[:, :, i]),
                            ((2, n, kv_heads, DIM), lambda t, i: t[i]), ((n, kv_heads, 2 * DIM), lambda t, i: t[..., i * DIM:(i + 1) * DIM])):
            both = torch.zeros(shape, dtype=dtype, device="cuda")
            kv.mpt_kv4_read(pages, *where, n, DIM, dtype=dtype, k_out=part(both, 0), v_out=part(both, 1))
            assert torch.equal(part(both, 0), k_want) and torch.equal(part(both, 1), v_want)
    kv.mpt_kv_check()
