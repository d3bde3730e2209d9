"""The model of the 4-bit cache on the CPU: what is put in comes back within half a step, and a planted
mistake in the layout does not."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import kv4_model as K


@pytest.mark.parametrize("dim", [8, 32, 40, 96, 256])
def test_round_trip(dim):
    rng = np.random.default_rng(dim)
    n = K.groups(dim)
    pages = rng.integers(0, 256, (3, 2, 2 * 288 * n), dtype=np.uint8)
    k, v = rng.standard_normal((2, 16, 2, dim)).astype(np.float32)
    k[3, 0] = 0
    v[5, 1] = 5.0
    k[6, 0, 0] = np.nan
    v[7, 0, 0] = np.inf
    for t in range(16):
        for h in range(2):
            K.put(pages, dim, 1, t, h, k[t, h], v[t, h])
    for x, got in zip((k, v), K.values(torch.from_numpy(pages), dim)):
        want = np.clip(np.nan_to_num(x, nan=0.0, posinf=3360.0), -3360, 3360).astype(np.float64)
        pad = np.pad(want, ((0, 0), (0, 0), (0, 32 * n - dim)), mode="edge") if dim % 32 else want
        g = pad.reshape(16, 2, n, 32)
        span = np.maximum((g.max(-1) - g.min(-1)) / 15, np.abs(g).max(-1) / 120)
        step = np.maximum(span, 2.0 ** -18) * 9 / 8  # rounded up to four bits: at most 9/8 of it
        err = np.abs(got[1].numpy().astype(np.float64) - want)
        assert (err <= np.repeat(step, 32, -1)[..., :dim] * (0.5 + 1e-6)).all()
    half = values_with_tokens_exchanged(pages, dim)
    assert np.abs(half - v)[np.isfinite(v) & (np.abs(v) < 100)].max() > 0.5


def values_with_tokens_exchanged(pages, dim):
    n = K.groups(dim)
    t = pages.reshape(3, 2, 2, 288 * n).copy()
    c = t[..., 144 * n:272 * n].reshape(3, 2, 2, 4, 8 * n, 2, 2)
    t[..., 144 * n:272 * n] = c[..., ::-1, :].reshape(3, 2, 2, -1)
    return np.nan_to_num(K.values(torch.from_numpy(t.reshape(pages.shape)), dim)[1][1].numpy())
