"""mpt_kv_merge refuses results that overlap what other threads still read; no GPU is needed for it."""

import struct

import pytest

from paper_2609_13692_gb300 import build as B

pytest.importorskip("torch")

ROWS, DIM = 8, 64
OUT, LSE = ROWS * DIM * 2, ROWS * 4  # bytes of a part
O1, O2, L1, L2, FREE = 1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20


@pytest.fixture(scope="module")
def merge():
    B.build()
    from paper_2609_13692_gb300 import mpt as M

    lib = M.load()
    return lambda out, lse, rows=ROWS: lib.mpt_kv_merge(struct.pack("@2P", O1, O2), struct.pack("@2P", L1, L2), 2, rows, DIM, 0, out, lse, 0)


@pytest.mark.parametrize("out,lse", [
    (FREE, L1), (FREE, L2), (FREE, L1 + 4), (FREE, L2 - 4), (FREE, L1 + LSE - 4), (FREE, L1 - LSE + 4),  # lse over a part's
    (O1 + 16, FREE), (O2 - 16, FREE), (O1 + OUT - 16, FREE), (O1 - OUT + 16, FREE),  # out over a part's, not the same
    (L1, FREE), (L2 - OUT + 16, FREE), (FREE, O1 + 16), (FREE, O2 + OUT - 4), (FREE, FREE), (FREE, FREE + OUT - 4), (FREE, FREE - LSE + 4),
])
def test_overlaps_are_refused(merge, out, lse):
    assert merge(out, lse) == 1
    assert merge(out, lse, rows=0) == 0  # nothing is read or written
