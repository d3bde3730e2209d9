"""Lengths that reach past the tensors: attention clamps them; writes, and codes read back, take them as they
are, and drop what lies outside.  Compared with calls whose lengths are in range, and with the plain models."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import kv4_model as K
from tests.test_kv4_gpu import BF16, args, kv, make, places  # noqa: F401

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32)
BEYOND = [0, 1, 41, 44]


@pytest.mark.parametrize("last", [50, 64, 2 ** 31 - 1])
@pytest.mark.parametrize("hint", [1, 40])
@pytest.mark.parametrize("dim", [64, 256])
def test_attention_clamps_offsets(kv, dim, hint, last):  # noqa: F811
    """The last offset beyond the tokens: as the number of tokens itself, in every row."""
    c = make(21, [1, 40, 3, 5], [60, 64, 9, 30], 4, 2, dim, 16, BF16)
    assert c["at"].tolist() == BEYOND + [49]
    want = kv.mpt_kv4_attend(*args(c), max_q_len=hint)
    got = kv.mpt_kv4_attend(*args(c)[:3], torch.tensor(BEYOND + [last], **I32, device="cuda"), c["lens"], max_q_len=hint)
    kv.mpt_kv_check()
    assert not bool(torch.isneginf(want[1]).any())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("last,lens", [(50, [60, 64, 9, 30]), (60, [60, 64, 9, 30]), (49, [60, 85, 9, 90]), (2 ** 31 - 1, [60, 64, 9, 2 ** 31 - 1])])
def test_writes_take_lengths_as_they_are(kv, last, lens):  # noqa: F811
    """Token t of request i stands at kv_lens[i] - (q_offsets[i + 1] - q_offsets[i]) + its place there, whatever the
    tensors hold: in 16 bits, turned, as codes, and read back."""
    c = make(22, [1, 40, 3, 5], [60, 64, 9, 30], 4, 2, 64, 16, BF16)
    n_pages, n = len(c["pages"]), 49
    at, lens = torch.tensor(BEYOND + [last], **I32, device="cuda"), torch.tensor(lens, **I32, device="cuda")
    where = c["table"], at, lens
    mine = places(*where, 16, n, n_pages)
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((n, 2, 64), generator=gen, device="cuda").to(BF16) for _ in range(2))
    turns = torch.from_numpy(K.angles(85, 64)).cuda()
    pool = torch.zeros((2, 2, n_pages, 16, 2, 64), dtype=BF16, device="cuda")
    kv.mpt_kv_write(k, v, pool[0, 0], pool[0, 1], *where)
    q = kv.mpt_kv_write_rotated(k, v, turns, pool[1, 0], pool[1, 1], *where, q=c["q"])
    kv.mpt_kv4_write(k, v, c["pages"], *where)
    got = kv.mpt_kv4_read(c["pages"], *where, n, 64, dtype=torch.float32)
    kv.mpt_kv_check()
    row = np.array([p for _, p, _ in mine])
    turned, q_turned = (torch.from_numpy(K.turned(x.float().cpu().numpy(), turns.cpu().numpy(), row, 64, False)).to(BF16) for x in (k, c["q"]))
    assert torch.equal(q.cpu(), q_turned)
    want, held = torch.zeros_like(pool, device="cpu"), K.values(c["pages"].cpu(), 64)
    for t, (_, pos, page) in enumerate(mine):
        if page < 0:
            assert not got[0][t].any() and not got[1][t].any()
            continue
        want[0, 0, page, pos % 16], want[0, 1, page, pos % 16] = k[t].cpu(), v[t].cpu()
        if pos < 85:  # else a position without a row
            want[1, 0, page, pos % 16], want[1, 1, page, pos % 16] = turned[t], v[t].cpu()
        assert torch.equal(got[0][t].cpu(), held[0][page, pos % 16]) and torch.equal(got[1][t].cpu(), held[1][page, pos % 16])
    assert torch.equal(pool.cpu(), want)
