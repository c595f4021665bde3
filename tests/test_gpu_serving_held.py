"""Appends behind rows that a page holds already, where only some of a page's waves have new rows."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import serving_oracle as O
from tests.test_gpu_serving import (DT, _gpu, batch_of, check_append, f64, make_cache, positions, randn,  # noqa: F401
                                    state, table_of)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,size,heads", [
    ("bf16", 128, 128, 8), ("bf16", 128, 64, 8), ("bf16", 64, 128, 5), ("bf16", 32, 64, 3), ("f32", 128, 64, 8),
    ("f32", 64, 128, 2)])
@pytest.mark.parametrize("turned", [False, True])
def test_held_rows_move_to_a_grown_scale(dtype, d, size, heads, turned):
    """Pages that hold all but a few of their rows, whose scales every appended row grows: the waves that hold
    earlier rows alone have none of the new ones, and round theirs again with the scale that the page had."""
    held = [size - 1, size - 3, 2 * size - 5, size // 2 + 1, 3 * size - 2, size - 1, 5, size - 9]
    lens = [40] * len(held)
    table, n_pages = table_of(np.random.default_rng(11), lens, held, size)
    cache = make_cache(heads, size, d, n_pages, table, seed=5)
    batch, cu = batch_of(lens, held)
    # louder than 127 of the held scales (0.04 at most) in every row and head
    k, v = ((randn(s, sum(lens), heads, d) * 8).to(DT[dtype]) for s in (1, 2))
    turns = scd.scd_rotary_table(scd.Rotary(d, 1e4), 512) if turned else None
    kx = O.rotate(f64(k), positions(lens, held), O.frequencies(d, 1e4)) if turned else f64(k)
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v, turns)
    check_append(cache, before, table, cu, held, (kx, f64(v)))
    for old, new in zip((before[0][1], before[1][1]), (f64(cache.k_scales), f64(cache.v_scales))):
        first = [table[b, h // size] for b, h in enumerate(held)]
        assert np.all(new[first] > old[first])


def test_a_long_batch_behind_held_rows():
    """Several heads of both branches a workgroup, every request's first page held in part: the append of all
    requests at once leaves what the appends of one request after another do."""
    size, heads, d = 64, 8, 128
    held = [1 + 7 * i % 63 for i in range(24)]
    lens = [300 + 11 * i for i in range(24)]
    table, n_pages = table_of(np.random.default_rng(12), lens, held, size)
    together, alone = (make_cache(heads, size, d, n_pages, table, seed=6) for _ in range(2))
    batch, cu = batch_of(lens, held)
    k, v = ((randn(s, sum(lens), heads, d) * 8).bfloat16() for s in (1, 2))
    scd.scd_cache_append(together, batch, k, v)
    for b in range(24):
        one = scd.PagedCache(alone.k_pages, alone.v_pages, alone.k_scales, alone.v_scales,
                             alone.page_table[b:b + 1].contiguous())
        part, _ = batch_of([lens[b]], [held[b]])
        scd.scd_cache_append(one, part, k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]])
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        assert torch.equal(getattr(together, name), getattr(alone, name)), name
