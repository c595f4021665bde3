"""Attention at the last positions that a cache can hold, where indices come close to 31 bits."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from tests.test_gpu_serving import DT, EPS, _gpu, f64, ints, make_cache, randn  # noqa: F401

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 64  # positions from here on are left out
SIZE = 128


def attended(cache, table, q, pos, scale):
    """Rows q [heads, d] of one request at position pos over the few pages that are no holes, in fp64."""
    heads, d = cache.n_kv_heads, cache.head_dim
    group = q.shape[0] // heads
    cols = np.nonzero(table >= 0)[0]
    at = (cols[:, None] * SIZE + np.arange(SIZE)).ravel()
    seen = (at <= pos) & (at < MOST)
    wide = lambda p, s: (f64(p)[table[cols]] * f64(s)[table[cols]][:, :, None, None]).transpose(1, 0, 2, 3).reshape(heads, -1, d)[:, seen]  # noqa: E731
    k, v = wide(cache.k_pages, cache.k_scales), wide(cache.v_pages, cache.v_scales)
    out, mass, reach = (np.zeros(q.shape) for _ in range(3))
    for i in range(q.shape[0]):
        s = scale * (k[i // group] @ q[i])
        p = np.exp(s - s.max())
        p /= p.sum()
        out[i], mass[i] = p @ v[i // group], p @ np.abs(v[i // group])
        reach[i] = scale * (np.abs(k[i // group]) @ np.abs(q[i])).max()
    return out, mass, reach


@pytest.mark.parametrize("dtype,d,tokens,heads", [("bf16", 32, 1, 2), ("f32", 64, 1, 1), ("bf16", 128, 3, 4),
                                                  ("bf16", 64, 130, 1)])
def test_attend_at_the_last_positions(dtype, d, tokens, heads):
    """One request whose table names all of 2^31 positions, nearly all of them holes: a few pages at its start, in
    the middle and at its end hold rows.  Rows of a few tokens, and of a prompt, around the last position."""
    table = np.full(2 ** 31 // SIZE, -1, dtype=np.int32)
    for i, col in enumerate((0, 7, 8, 2 ** 23, 2 ** 24 - 160, 2 ** 24 - 3, 2 ** 24 - 2, 2 ** 24 - 1)):
        table[col] = i + 1
    cache = make_cache(1, SIZE, d, 10, [[0]], seed=3)
    cache = scd.PagedCache(cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales,
                           torch.from_numpy(table).cuda().view(1, -1))
    first = MOST - 1 - tokens // 2
    q = randn(8, tokens, heads, d).to(DT[dtype])
    out = torch.full_like(q, float("nan"))
    scd.scd_cache_attend(cache, scd.Batch(tokens, ints([0, tokens]), ints([first])), q, out)
    # as in the tests of ordinary lengths: scores off by 2^-19 of scale * sum |q||k|, bf16 weights of 11 bits
    for t in sorted({0, tokens // 2, tokens - 1}):
        want, mass, reach = attended(cache, table, f64(q[t]), first + t, d ** -0.5)
        rel = 2 * 2.0 ** -19 * reach + 2.0 ** -18 + (2.0 ** -10 if dtype == "bf16" else 0.0)
        assert np.all(np.abs(f64(out[t]) - want) <= rel * mass + 0.51 * EPS[dtype] * np.abs(want)), t
