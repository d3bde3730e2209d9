"""The operators as they are used together (examples/serve_layout.py): a laid-out group served from the
paged cache computes exactly the layout's cost, and every output is the attention of the whole prompt."""

import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")

from tests import kv_model as M

pytestmark = pytest.mark.gpu

EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    B.build()
    sys.path.insert(0, EXAMPLES)
    import serve_layout

    return serve_layout


def bounds(layer, tokens):
    """(attention of the whole prompt in 64 bits, its bound) per token."""
    q, k, v = layer.project(tokens)
    n = len(tokens)
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = -(-n // 256)
    pad = torch.zeros((2, pages * 256, *k.shape[1:]), dtype=k.dtype, device="cuda")
    pad[0, :n], pad[1, :n] = k, v
    pad = pad.view(2, pages, 256, *k.shape[1:])
    out, _, tol, _ = M.attend(q, pad[0], pad[1], torch.arange(pages, **i32)[None], torch.tensor([0, n], **i32),
                              torch.tensor([n], **i32), True, 1 / math.sqrt(q.shape[2]))
    return out, tol


@pytest.mark.parametrize("m,page_size,heads,kv_heads,head_dim", [(12, 16, 16, 4, 128), (7, 32, 8, 8, 64), (9, 8, 12, 2, 96)])
def test_layout_is_served(example, m, page_size, heads, kv_heads, head_dim):
    got = example.serve(m=m, page_size=page_size, heads=heads, kv_heads=kv_heads, head_dim=head_dim)
    assert got["prefilled"] == got["cost"] < got["tokens"]
    for r, (keep, out) in got["outputs"].items():
        want, tol = bounds(got["layer"], example.prompt_tokens(got["strings"][r], got["weights"]))
        assert bool(((out.double() - want[keep:]).abs() <= tol[keep:]).all()), r
    for whole, merged in got["both"]:
        # each part rounded once and weighed, the merge once more: a few roundings of values of this size
        assert float((whole.double() - merged.double()).abs().max()) <= 8 * M.UNIT[whole.dtype] * float(whole.abs().max())
    assert got["last_after"] == got["live"] - 1 <= got["last_before"]
    assert torch.equal(got["apart"], got["together"])
