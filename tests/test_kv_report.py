"""What mpt_kv_check tells (csrc/kv_report.h), compiled for the host: an event that a kernel counts at any
moment is told of by some call, and by no later one again."""

import ctypes
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "%s/paper_2609_13692_gb300/csrc/kv_report.h"
extern "C" mpt::Reported* make() { return new mpt::Reported; }
extern "C" int news(mpt::Reported* r, int device, uint32_t count) { return r->news(device, count); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    at = tmp_path_factory.mktemp("report")
    (at / "r.cpp").write_text(SOURCE % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(at / "r.so"), str(at / "r.cpp")],
                   check=True)
    lib = ctypes.CDLL(str(at / "r.so"))
    lib.make.restype = ctypes.c_void_p
    lib.news.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32]
    return lib


def test_every_event_is_told_once(lib):
    """All orders of two calls, each a read and an answer, and two events: a third call afterwards knows of none,
    every event was told of by a call that read after it, and no call tells of what was told before it read."""
    steps = ["e", "e", "read0", "news0", "read1", "news1"]
    for order in set(itertools.permutations(steps)):
        if order.index("read0") > order.index("news0") or order.index("read1") > order.index("news1"):
            continue
        r, count, read, told = lib.make(), 0, {}, 0
        for s in order:
            if s == "e":
                count += 1
            elif s.startswith("read"):
                read[s[4]] = (count, told)
            elif lib.news(r, 0, read[s[4]][0]):
                assert read[s[4]][0] > read[s[4]][1], order
                told = max(told, read[s[4]][0])
            else:
                assert told >= read[s[4]][0], order
        assert lib.news(r, 0, count) == (told < count), order
        assert lib.news(r, 0, count) == 0


def test_devices_and_wrap(lib):
    r = lib.make()
    assert lib.news(r, 1, 3) == 1 and lib.news(r, 0, 1) == 1 and lib.news(r, 1, 3) == 0 and lib.news(r, 1, 4) == 1
    assert lib.news(r, 1, 2) == 0  # an older read
    assert lib.news(r, 2, 1 << 30) == 1 and lib.news(r, 2, 1 << 31) == 1 and lib.news(r, 2, 3 << 30) == 1 and lib.news(r, 2, 5) == 1
    assert lib.news(r, 64, 0) == 0 and lib.news(r, 64, 1) == 1


def test_nothing_clears_the_counts():
    """No call writes the kernels' counts from the host."""
    csrc = os.path.join(ROOT, "paper_2609_13692_gb300", "csrc")
    for name in ("k_attend_few.cu", "k_attend_tile.cu", "mpt_kv.cu", "k_kv_pages.cu", "kv_internal.cuh"):
        text = open(os.path.join(csrc, name)).read()
        assert "cudaMemsetAsync" not in text and "cudaMemcpyToSymbol" not in text, name
