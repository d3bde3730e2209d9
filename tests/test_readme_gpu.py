"""The README's calls of the paged cache, as they are written there, on tensors of their shapes."""

import os
import re
import textwrap

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def blocks():
    """The indented blocks that call the cache, in order."""
    text = open(os.path.join(ROOT, "README.md")).read()
    found = re.findall(r"(?:^    .*\n)+", text, re.M)
    return [textwrap.dedent(b) for b in found if "kv.mpt_kv" in b]


def test_calls_of_the_cache():
    """In both caches keys and queries are turned once by their positions, and attention is over what was written."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_13692_gb300 import build as B

    B.build()
    from paper_2609_13692_gb300 import kv
    from tests import kv4_model as K

    gen = torch.Generator(device="cuda").manual_seed(11)
    page_size, kv_heads, head_dim, n_pages, heads, n = 16, 2, 64, 12, 4, 9
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.full((3, 4), -1, **i32)
    table[0, :2] = torch.tensor([5, 2], **i32)
    refs = torch.zeros(n_pages, **i32)
    refs[[5, 2]] = 1
    pool = torch.randn((1, n_pages, 2, page_size, kv_heads, head_dim), generator=gen, device="cuda").bfloat16()
    q = torch.randn((2 * n, heads, head_dim), generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn((2 * n, kv_heads, head_dim), generator=gen, device="cuda").bfloat16() for _ in range(2))
    turns = torch.from_numpy(K.angles(64, head_dim)).cuda()
    space = dict(torch=torch, page_size=page_size, kv_heads=kv_heads, head_dim=head_dim, n_pages=n_pages, table=table,
                 lens=torch.tensor([29, 0, 0], **i32), refs=refs, pool=pool, q=q.clone(), k=k, v=v, turns=turns,
                 src_rows=torch.tensor([0, 0], **i32), dst_rows=torch.tensor([1, 2], **i32), keep=torch.tensor([29, 20], **i32),
                 rows=torch.tensor([1, 2], **i32), new_tokens=torch.tensor([n, n], **i32), q_offsets=torch.tensor([0, 0, n, 2 * n], **i32))
    first, *rest = blocks()
    exec(first, space)
    kv.mpt_kv_check()
    where = space["table"], space["q_offsets"], space["lens"]
    plain = pool.clone()
    want = kv.mpt_kv_attend(q, plain[0, :, 0], plain[0, :, 1], *where)
    assert space["lens"].tolist() == [29, 38, 29] and torch.equal(space["out"], want[0]) and torch.equal(space["lse"], want[1])

    pos = torch.tensor([*range(29, 38), *range(20, 29)])
    turned = torch.from_numpy(K.turned(q.float().cpu().numpy(), turns.cpu().numpy(), pos.numpy(), head_dim, False)).bfloat16().cuda()
    pages = torch.zeros((n_pages, kv_heads, kv.mpt_kv4_page_bytes(page_size, head_dim)), dtype=torch.uint8, device="cuda")
    kv.mpt_kv4_write(k, v, pages, *where, rotation=turns)
    wide = pool.clone()
    kv.mpt_kv_write_rotated(k, v, turns, wide[0, :, 0], wide[0, :, 1], *where)
    in_codes = kv.mpt_kv4_attend(turned, pages, *where)
    in_16 = kv.mpt_kv_attend(turned, wide[0, :, 0], wide[0, :, 1], *where)
    handed = []  # queries, as each attention gets them
    calls = {name: getattr(kv, name) for name in ("mpt_kv_attend", "mpt_kv4_attend")}
    results = {}

    def watched(name):
        def call(x, *more, **named):
            handed.append(x.clone())
            results[name] = calls[name](x, *more, **named)
            return results[name]
        return call

    with pytest.MonkeyPatch.context() as m:
        for name in calls:
            m.setattr(kv, name, watched(name))
        for block in rest:
            exec(block, space)
    kv.mpt_kv_check()
    assert torch.equal(space["pages"], pages) and torch.equal(pool, wide)
    assert torch.equal(space["q"], q)  # the unturned ones keep their name
    assert set(results) == set(calls) and all(torch.equal(x, turned) for x in handed)
    for name, right in (("mpt_kv4_attend", in_codes), ("mpt_kv_attend", in_16)):
        assert all(torch.equal(a, b) for a, b in zip(results[name], right)), name
