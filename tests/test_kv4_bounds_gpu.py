"""The turned writes and the 4-bit cache in the bounds-checked build (compiled with MPT_BOUNDS): the tests of
ragged, holed, empty and out-of-range cases run on that library in a child process and end without a report."""

import os
import re
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

from tests.test_kv_bounds_gpu import CHILD, ROOT

CASES = ("writes or codes or turned or page_sizes or holes or see_nothing or many_requests or behind_the_last or decrease "
         "or served_like or out_of_range or more_items or long_keys or large_groups or more_requests or last_of_32")


@pytest.mark.gpu
def test_bounds_checked_build_runs_clean():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    env = dict(os.environ, MPT_LIBRARY=str(B.build(bounds=True)))
    files = ["tests/test_kv4_gpu.py", "tests/test_kv4_edges_gpu.py"]
    p = subprocess.run([sys.executable, "-c", CHILD, CASES, *files], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert p.returncode == 0, (p.stdout[-4000:], p.stderr[-2000:])
    assert "BOUNDS_OK" in p.stdout and " passed" in p.stdout


@pytest.mark.parametrize("name,kernels", [("k_kv_append.cu", ["k_kv_append", "k_kv4_read"]),
                                          ("k_attend4_few.cu", ["k_attend4_few", "k_attend4_few_join"]), ("k_attend_tile.cu", ["widen_codes"])])
def test_kernels_that_index_by_device_data_check(name, kernels):
    """Each kernel that takes indices from device data has a check of its own."""
    text = open(os.path.join(ROOT, "paper_2609_13692_gb300", "csrc", name)).read()
    starts = [m.start() for m in re.finditer(r"^(?:template <[^\n]*>\n)?(?:__global__|__device__)", text, re.M)] + [len(text)]
    parts = [text[a:b] for a, b in zip(starts, starts[1:])]
    for k in kernels:
        own = [p for p in parts if re.match(r"[^{;]*\b%s\(" % k, p)]
        assert own and "KV_BAD(" in own[0], k
