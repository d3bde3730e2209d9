"""The turned writes and the 4-bit cache without a GPU: host-side checks come before any CUDA call and
return the documented statuses; calls with nothing to do succeed; what the binding refuses."""

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
S = struct.pack("@2q", 64, 64)


def cache(**more):
    from paper_2609_13692_gb300 import kv

    d = dict(k=A, v=A, k0=1024, k1=64, k2=64, v0=1024, v1=64, v2=64, type=0, n_pages=10, page=16, heads=1, dim=64, batch=2,
             table=A, stride=5, width=5, offsets=A, lens=A)
    d.update(more)
    return kv._CACHE.pack(*d.values())


def cache4(**more):
    from paper_2609_13692_gb300 import kv

    d = dict(pages=A, s0=1152 * 2, s1=1152, n_pages=10, page=16, heads=2, dim=64, batch=2, table=A, stride=5, width=5, offsets=A, lens=A)
    d.update(more)
    return kv._CACHE4.pack(*d.values())


def turn(**more):
    from paper_2609_13692_gb300 import kv

    d = dict(table=A, stride=64, rows=100, rot=64, adjacent=0, heads=2, positions=0, q=A, q_out=A, q0=128, q1=64, o0=128, o1=64)
    d.update(more)
    return kv._TURN.pack(*d.values())


def rotated(lib, c=None, u=None, k=A, v=A, ks=S, vs=S, tokens=2):
    return lib.mpt_kv_write_rotated(cache() if c is None else c, turn() if u is None else u, k, ks, v, vs, tokens, 0)


def write(lib, c=None, u=None, type=0, k=A, v=A, ks=S, vs=S, tokens=2):
    return lib.mpt_kv4_write(cache4() if c is None else c, u, type, k, ks, v, vs, tokens, 0)


def read(lib, c=None, type=0, k=A, v=A, ks=S, vs=S, tokens=2):
    return lib.mpt_kv4_read(cache4() if c is None else c, type, k, ks, v, vs, tokens, 0)


def attend(lib, c=None, type=0, q=A, tokens=2, heads=4, hint=0, scale=0.1, out=A, ws=A, ws_bytes=1 << 40, qs=(256, 64), os=(256, 64), lse=A):
    return lib.mpt_kv4_attend(cache4() if c is None else c, type, q, struct.pack("@2q", *qs), tokens, heads, hint, 1, scale, out,
                              struct.pack("@2q", *os), lse, ws, ws_bytes, 0)


def test_nothing_to_do(lib):
    none = cache4(batch=0, table=0, offsets=0, lens=0)
    assert rotated(lib, tokens=0) == 0 and rotated(lib, cache(batch=0, table=0, offsets=0, lens=0)) == 0
    for call in (write, read, attend):
        assert call(lib, tokens=0) == 0 and call(lib, none) == 0
    assert write(lib, u=turn(), tokens=0) == 0


def test_page_bytes(lib):
    n = ctypes.c_int64()
    for page, dim, want in ((8, 8, 288), (16, 128, 2304), (256, 256, 32 * 2304), (32, 80, 4 * 864)):
        assert lib.mpt_kv4_page_bytes(page, dim, ctypes.byref(n)) == 0 and n.value == want
    for page, dim in ((4, 64), (24, 64), (512, 64), (16, 0), (16, 12), (16, 264)):
        assert lib.mpt_kv4_page_bytes(page, dim, ctypes.byref(n)) == 1
    assert lib.mpt_kv4_page_bytes(16, 64, None) == 1


@pytest.mark.parametrize("more,status", [
    (dict(pages=0), 1), (dict(pages=A + 8), 1), (dict(n_pages=0), 1), (dict(page=4), 1), (dict(page=24), 1), (dict(page=512), 1),
    (dict(heads=0), 1), (dict(dim=0), 1), (dict(dim=12), 1), (dict(dim=264), 2), (dict(heads=1025), 2), (dict(batch=-1), 1),
    (dict(batch=(1 << 20) + 1), 2), (dict(width=0), 1), (dict(stride=4), 1), (dict(table=0), 1), (dict(offsets=0), 1),
    (dict(lens=0), 1), (dict(table=A + 2), 1), (dict(s0=1136), 1), (dict(s1=1136), 1), (dict(s0=1160 * 2 + 8), 1), (dict(s1=1160), 1),
    (dict(s1=0), 1), (dict(s0=-2304), 1), (dict(s0=1 << 38), 1), (dict(width=1 << 28, stride=1 << 28), 2),
])
def test_cache_checks(lib, more, status):
    for call in (write, read, attend):
        assert call(lib, cache4(**more)) == status, call


@pytest.mark.parametrize("more,status", [
    (dict(table=0), 1), (dict(table=A + 4), 1), (dict(rows=0), 1), (dict(rot=0), 1), (dict(rot=-16), 1), (dict(rot=8), 1), (dict(rot=24), 1),
    (dict(rot=80), 1), (dict(rot=4, adjacent=1), 1), (dict(rot=72, adjacent=1), 1), (dict(stride=60), 1), (dict(stride=66), 1),
    (dict(positions=A + 2), 1), (dict(q_out=0), 1), (dict(q=A + 8), 1), (dict(q_out=A + 8), 1), (dict(heads=0), 1),
    (dict(heads=(1 << 17) + 1), 2), (dict(q0=60), 1), (dict(q1=0), 1), (dict(o0=-128), 1), (dict(o0=256), 1), (dict(o1=72), 1),
])
def test_turn_checks(lib, more, status):
    assert rotated(lib, u=turn(**more)) == status
    assert write(lib, u=turn(**more)) == status


def test_new_token_checks(lib):
    assert rotated(lib, c=0) == 1 and rotated(lib, u=0) == 1
    for call in (rotated, write, read):
        assert call(lib, k=0) == 1 and call(lib, v=0) == 1 and call(lib, k=A + 8) == 1 and call(lib, v=A + 2) == 1
        assert call(lib, ks=None) == 1 and call(lib, vs=struct.pack("@2q", 60, 64)) == 1
        assert call(lib, tokens=-1) == 1 and call(lib, tokens=1 << 31) == 2
    assert write(lib, type=2) == 1 and write(lib, type=-1) == 1 and read(lib, type=3) == 1 and read(lib, type=-1) == 1


def test_attend_checks(lib):
    assert attend(lib, 0) == 1 and attend(lib, type=2) == 1 and attend(lib, type=-1) == 1
    assert attend(lib, heads=0) == 1 and attend(lib, heads=3) == 1
    assert attend(lib, heads=258) == 2 and attend(lib, heads=256, tokens=1 << 24) == 2
    assert attend(lib, tokens=-1) == 1 and attend(lib, tokens=1 << 31) == 2
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert attend(lib, scale=scale) == 1
    assert attend(lib, hint=-1) == 1
    assert attend(lib, q=0) == 1 and attend(lib, q=A + 4) == 1 and attend(lib, out=0) == 1 and attend(lib, lse=A + 2) == 1
    assert attend(lib, qs=(252, 64)) == 1 and attend(lib, os=(256, 0)) == 1
    assert lib.mpt_kv4_attend_workspace_bytes(None) == 1


def test_binding_refuses():
    from paper_2609_13692_gb300 import kv

    i = torch.zeros(2, dtype=torch.int32)
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    p = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    u = torch.zeros((3, 4, 1152), dtype=torch.uint8)
    r = torch.zeros((9, 64))
    for call in (lambda: kv.mpt_kv4_attend(x, u, i[None], i, i[:1]), lambda: kv.mpt_kv4_write(x, x, u, i[None], i, i[:1]),
                 lambda: kv.mpt_kv4_read(u, i[None], i, i[:1], 2, 64),
                 lambda: kv.mpt_kv_write_rotated(x[:, :2], x[:, :2], r, p, p, i[None], i, i[:1])):
        with pytest.raises(ValueError):  # host tensors
            call()


def test_binding_packs():
    """Shapes and types that the binding turns down, and what it packs, on host tensors past the device check."""
    from paper_2609_13692_gb300 import kv

    i = torch.zeros(2, dtype=torch.int32)
    u = torch.zeros((3, 4, 1152), dtype=torch.uint8)
    got = kv._CACHE4.unpack(kv._cache4(u, i[None], i, i[:1], 64))
    assert got[1:8] == (4608, 1152, 3, 16, 4, 64, 1) and got[9:11] == (2, 2)
    for pages, dim in ((u[:, :, :1000], 64), (u, 96), (u.int(), 64), (u.transpose(1, 2), 64), (u[0], 64), (u[:, :, :0], 64)):
        with pytest.raises(ValueError):
            kv._cache4(pages, i[None], i, i[:1], dim)
    with pytest.raises(ValueError):
        kv._cache4(u, i[None], i[:1], i[:1], 64)
    with pytest.raises(ValueError):
        kv._cache4(u, i[None].long(), i, i[:1], 64)
