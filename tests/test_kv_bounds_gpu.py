"""The paged-cache operators in the bounds-checked build (compiled with MPT_BOUNDS): their kernels count and skip
any index that is out of range, and mpt_kv_check reports it.  The tests of ragged, holed, empty and out-of-range
cases run on that library in a child process (MPT_LIBRARY), which has to end without a report."""

import os
import re
import subprocess
import sys
import textwrap

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CASES = ("page_sizes or holes or see_nothing or not_finite or many_requests or long_keys or out_of_range or noted_values "
         "or decrease or large_groups or more_requests or write or bookkeeping or copy_pages or merge or layout_is_served")

CHILD = textwrap.dedent(r"""
    import sys
    import pytest
    from paper_2609_13692_gb300 import kv, mpt

    mpt.load()
    assert mpt.mpt_build_info()["bounds_checked"], "not the bounds-checked library"
    rc = pytest.main(["-q", "-x", "-m", "gpu", "-p", "no:cacheprovider", "-k", sys.argv[1], *sys.argv[2:]])
    assert rc == 0, rc
    kv.mpt_kv_check()
    print("BOUNDS_OK")
""")


@pytest.mark.gpu
def test_bounds_checked_build_runs_clean():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    env = dict(os.environ, MPT_LIBRARY=str(B.build(bounds=True)))
    files = ["tests/test_kv_%s_gpu.py" % n for n in ("attend", "pages", "edges", "serving")]
    p = subprocess.run([sys.executable, "-c", CHILD, CASES, *files], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert p.returncode == 0, (p.stdout[-4000:], p.stderr[-2000:])
    assert "BOUNDS_OK" in p.stdout and " passed" in p.stdout


@pytest.mark.parametrize("name,kernels", [
    ("k_kv_pages.cu", ["k_kv_merge", "k_kv_write", "k_kv_copy_pages", "k_kv_book", "k_kv_compact"]),
    ("k_attend_few.cu", ["k_attend_few", "k_attend_few_join"]), ("k_attend_tile.cu", ["fill_list", "k_attend_tile", "k_attend_tile_join"])])
def test_kernels_that_index_by_device_data_check(name, kernels):
    """Each kernel that takes indices from device data has a check of its own, which the default build leaves out."""
    text = open(os.path.join(ROOT, "paper_2609_13692_gb300", "csrc", name)).read()
    starts = [m.start() for m in re.finditer(r"^(?:template <[^\n]*>\n)?(?:__global__|__device__)", text, re.M)] + [len(text)]
    parts = [text[a:b] for a, b in zip(starts, starts[1:])]
    for k in kernels:
        own = [p for p in parts if re.match(r"[^{;]*\b%s\(" % k, p)]
        assert own and "KV_BAD(" in own[0], k
    head = open(os.path.join(ROOT, "paper_2609_13692_gb300", "csrc", "kv_internal.cuh")).read()
    assert "#else\n#define KV_BAD(counts, ok) false\n" in head
