"""How much of a bf16 query the attention over 4-bit codes sees beside a larger element of its row."""

import pytest

torch = pytest.importorskip("torch")

from tests import kv4_model as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    B.build()
    from paper_2609_13692_gb300 import kv as K

    return K


@pytest.mark.parametrize("hint", [1, 32])
@pytest.mark.parametrize("dim", [32, 128, 256])
@pytest.mark.parametrize("e", [-40, 0, 40])
def test_small_elements_beside_a_large_one(kv, dim, e, hint):
    """Rows with an element in [2^e, 2^(e+1)) that the key has a 0 for, and one of each significand 2^-j as large:
    seen as it is down to j = 17, and to 2^(e-25) below.

    A row's lse is its one score, about 4 to 8 by the choice of the scale.  In powers of two it is below 12; the
    scale's and the products' roundings take 4 x 12 x 2^-24 of it, the exponential 2^-21, its argument, the
    logarithm and two sums of numbers below 16 half a step of 2^-20 each, the logarithm another: 2^-18 together."""
    i32 = dict(dtype=torch.int32, device="cuda")
    n, heads = 32, 4  # 128 significands of 8 bits
    new = torch.zeros((1, 1, dim), dtype=torch.bfloat16, device="cuda")
    new[0, 0, dim - 1] = 3000
    pages = torch.zeros((1, 1, kv.mpt_kv4_page_bytes(8, dim)), dtype=torch.uint8, device="cuda")
    where = torch.zeros((1, 1), **i32), torch.tensor([0, 1], **i32), torch.tensor([1], **i32)
    kv.mpt_kv4_write(new, new, pages, *where)
    key = K.values(pages, dim)[0][0, 0, 0]
    assert float(key[dim - 1]) > 2500 and int((key != 0).sum()) == 1
    small = (1 + torch.arange(n * heads, device="cuda").double() / 128).view(n, heads)
    at = torch.tensor([0, n], **i32)
    for j in (1, 10, 14, 15, 16, 17, 18, 20, 23):
        q = torch.zeros((n, heads, dim), dtype=torch.bfloat16, device="cuda")
        q[..., 0] = 1.9921875 * 2.0 ** e
        q[..., dim - 1] = (small * 2.0 ** (e - j)).bfloat16()
        assert torch.equal(q[..., dim - 1].double(), small * 2.0 ** (e - j))
        scale = 4 / (2.0 ** (e - j) * float(key[dim - 1]))
        _, lse = kv.mpt_kv4_attend(q, pages, where[0], at, where[2], causal=False, scale=scale, max_q_len=hint)
        kv.mpt_kv_check()
        bound = 0.0 if j <= 17 else scale * 2.0 ** (e - 25) * float(key[dim - 1])
        assert float((lse.double() - 4 * small).abs().max()) <= bound + 2.0 ** -18, j
