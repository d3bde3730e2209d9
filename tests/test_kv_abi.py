"""mpt_kv.h without a GPU: the host-side checks come before any CUDA call and return the documented
statuses; calls with nothing to do succeed."""

import ctypes
import math
import struct

import pytest

from paper_2609_13692_gb300 import build as B

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    B.build()
    from paper_2609_13692_gb300 import mpt as M

    return M.load()


A = 1 << 20  # an address that nothing reads: every call below returns before it would


def cache(**more):
    d = dict(k=A, v=A, k0=1024, k1=64, k2=64, v0=1024, v1=64, v2=64, type=0, n_pages=10, page=16, heads=1, dim=64, batch=2,
             table=A, stride=5, width=5, offsets=A, lens=A)
    d.update(more)
    from paper_2609_13692_gb300 import kv

    return kv._CACHE.pack(*d.values())


def attend(lib, c=None, q=A, tokens=2, heads=4, hint=0, scale=0.1, out=A, ws=A, ws_bytes=1 << 40, qs=(256, 64), os=(256, 64), lse=A):
    return lib.mpt_kv_attend(cache() if c is None else c, q, struct.pack("@2q", *qs), tokens, heads, hint, 1, scale, out,
                             struct.pack("@2q", *os), lse, ws, ws_bytes, 0)


def test_nothing_to_do(lib):
    assert attend(lib, tokens=0) == 0
    assert attend(lib, cache(batch=0, table=0, offsets=0, lens=0)) == 0
    assert lib.mpt_kv_write(cache(), A, struct.pack("@2q", 64, 64), A, struct.pack("@2q", 64, 64), 0, 0) == 0
    ptrs = struct.pack("@2P", A, A)
    assert lib.mpt_kv_merge(ptrs, ptrs, 2, 0, 64, 0, A, A * 2, 0) == 0
    assert lib.mpt_kv_copy_pages(A, 1, 0, 4, 64, 64, A, A, 0, 0) == 0


@pytest.mark.parametrize("more,status", [
    (dict(k=0), 1), (dict(v=A + 8), 1), (dict(type=2), 1), (dict(type=-1), 1), (dict(n_pages=0), 1), (dict(page=4), 1),
    (dict(page=24), 1), (dict(page=512), 1), (dict(heads=0), 1), (dict(dim=0), 1), (dict(dim=12), 1), (dict(dim=264), 2),
    (dict(heads=1025), 2), (dict(batch=-1), 1), (dict(batch=(1 << 20) + 1), 2), (dict(width=0), 1), (dict(stride=4), 1),
    (dict(table=0), 1), (dict(offsets=0), 1), (dict(lens=0), 1), (dict(table=A + 2), 1), (dict(k1=63), 1), (dict(k1=0), 1),
    (dict(k0=-64), 1), (dict(v1=4), 1), (dict(width=1 << 28, stride=1 << 28), 2),
])
def test_cache_checks(lib, more, status):
    assert attend(lib, cache(**more)) == status
    s = struct.pack("@2q", 64, 64)
    assert lib.mpt_kv_write(cache(**more), A, s, A, s, 2, 0) == status


def test_attend_checks(lib):
    assert attend(lib, 0) == 1
    assert attend(lib, heads=0) == 1 and attend(lib, cache(heads=3, k2=64, v2=64), heads=4) == 1
    assert attend(lib, heads=129) == 2 and attend(lib, heads=128, tokens=1 << 24) == 2
    assert attend(lib, tokens=-1) == 1 and attend(lib, tokens=1 << 31) == 2
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert attend(lib, scale=scale) == 1
    assert attend(lib, hint=-1) == 1
    assert attend(lib, q=0) == 1 and attend(lib, q=A + 4) == 1 and attend(lib, out=0) == 1 and attend(lib, lse=A + 2) == 1
    assert attend(lib, qs=(252, 64)) == 1 and attend(lib, os=(256, 0)) == 1
    n = ctypes.c_size_t()
    for dim, status in ((0, 1), (12, 1), (264, 1)):
        assert lib.mpt_kv_attend_workspace_bytes(dim, ctypes.byref(n)) == status
    assert lib.mpt_kv_attend_workspace_bytes(64, None) == 1


def test_merge_checks(lib):
    def merge(n=2, rows=4, dim=64, type=0, outs=(A, A), lses=(A, A), out=A, lse=2 * A):
        return lib.mpt_kv_merge(struct.pack("@2P", *outs), struct.pack("@2P", *lses), n, rows, dim, type, out, lse, 0)

    assert merge(n=0) == 1 and merge(n=17) == 2 and merge(rows=-1) == 1 and merge(dim=4) == 1 and merge(dim=1032) == 2
    assert merge(type=3) == 1 and merge(outs=(A, 0)) == 1 and merge(lses=(A, A + 2)) == 1 and merge(out=A + 8) == 1
    assert merge(lse=A) == 1  # the sums of a part are read by several threads of its rows
    assert lib.mpt_kv_merge(None, None, 2, 4, 64, 0, A, A, 0) == 1


def test_book_checks(lib):
    from paper_2609_13692_gb300 import kv

    def book(**more):
        d = dict(table=A, stride=5, width=5, rows=8, lens=A, refs=A, n_pages=10, page=16)
        d.update(more)
        return kv._BOOK.pack(*d.values())

    def free(b, n=1, rows=A, status=A):
        return lib.mpt_kv_free(b, rows, n, status, 0)

    for more, status in ((dict(table=0), 1), (dict(stride=4), 1), (dict(width=0), 1), (dict(rows=0), 1), (dict(rows=(1 << 20) + 1), 2),
                         (dict(lens=0), 1), (dict(refs=A + 1), 1), (dict(n_pages=0), 1), (dict(n_pages=1 << 30), 2), (dict(page=20), 1),
                         (dict(width=1 << 28, stride=1 << 28), 2)):
        assert free(book(**more)) == status, more
    assert free(book(), n=-1) == 1 and free(book(), n=9) == 2 and free(book(), rows=0) == 1 and free(book(), status=0) == 1
    assert free(book(rows=1 << 15), n=16_385) == 2
    assert lib.mpt_kv_fork(book(), A, A, A, 1, A, A, A, 0) == 1  # one list for both pages of the pairs
    assert lib.mpt_kv_extend(book(), A, 0, 1, A, 0) == 1
    assert lib.mpt_kv_compact(book(), 0, A, A, 0) == 1


def test_copy_checks(lib):
    def copy(pool=A, planes=1, plane=0, n_pages=4, stride=64, size=64, src=A, dst=A, n=1):
        return lib.mpt_kv_copy_pages(pool, planes, plane, n_pages, stride, size, src, dst, n, 0)

    for more, status in ((dict(pool=0), 1), (dict(pool=A + 8), 1), (dict(planes=0), 1), (dict(n_pages=0), 1), (dict(n=-1), 1),
                         (dict(size=0), 1), (dict(size=24, stride=64), 1), (dict(stride=48), 1), (dict(stride=72), 1), (dict(plane=8), 1),
                         (dict(src=0), 1), (dict(dst=A + 1), 1), (dict(n_pages=1 << 30), 2), (dict(planes=1 << 17), 2)):
        assert copy(**more) == status, more


def test_binding_refuses_host_tensors():
    from paper_2609_13692_gb300 import kv

    i = torch.zeros(2, dtype=torch.int32)
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    p = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: kv.mpt_kv_attend(x, p, p, i[None], i, i[:1]), lambda: kv.mpt_kv_write(x[:, :2], x[:, :2], p, p, i[None], i, i[:1]),
                 lambda: kv.mpt_kv_merge([x, x], [x[..., 0].float()] * 2), lambda: kv.mpt_kv_free(i[None], i[:1], i, 16, i),
                 lambda: kv.mpt_kv_copy_pages(p[None], i, i)):
        with pytest.raises(ValueError):
            call()
