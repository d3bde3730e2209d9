"""mpt_kv_copy_pages counts pairs x planes x 16 KB pieces in 64 bits and refuses more; no GPU is needed for it."""

import pytest

from paper_2609_13692_gb300 import build as B

pytest.importorskip("torch")


def test_more_units_than_64_bits_count():
    B.build()
    from paper_2609_13692_gb300 import mpt as M

    lib, at = M.load(), 1 << 20

    def copy(planes, size, n):
        return lib.mpt_kv_copy_pages(at, planes, 0, 4, size, size, at, at, n, 0)

    # 2^30 - 1 pairs, 2^16 planes, pages of 4 GB: 2^64 - 2^34 pieces
    assert copy(1 << 16, 1 << 32, (1 << 30) - 1) == 2
    assert copy(1 << 16, 1 << 32, 1 << 28) == 2
    assert copy(1 << 16, 1 << 32, 0) == 0
