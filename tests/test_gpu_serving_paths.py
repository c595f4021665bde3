"""The layouts a call of the serving operators can take: whole and cut segments, shares of a prompt, long lists of
pages, many requests, shared workspaces, captured steps that grow from one layout's lengths into another's."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import serving_oracle as O
from tests.test_gpu_serving import (DT, EPS, _gpu, batch_of, check_append, check_attend, f64, ints,  # noqa: F401
                                    make_cache, positions, randn, state, table_of)

pytestmark = pytest.mark.gpu


def sampled(cache, table, cu, held, q, out, rows):
    """The given packed rows of a bf16 call against the oracle, request by request."""
    pages = [x.cpu().numpy() for x in (cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales)]
    for t in rows:
        b = int(np.searchsorted(cu, t, side="right")) - 1
        one = q[t:t + 1]
        want, mass, reach = O.attend(f64(one), *pages, table[b:b + 1], [0, 1], [held[b] + t - cu[b]], cache.head_dim ** -0.5)
        rel = 2 * 2.0 ** -19 * reach[..., None] + 2.0 ** -18 + 2.0 ** -10
        assert np.all(np.abs(f64(out[t:t + 1]) - want) <= rel * mass + 0.51 * EPS["bf16"] * np.abs(want)), t


@pytest.mark.parametrize("lens,held,heads,kv_heads,d", [
    ([2100], [15000], 32, 8, 128),   # no shares, and more groups of positions than one list holds
    ([300], [5000], 32, 8, 128),     # several shares of every tile
    ([64], [20000], 4, 1, 128),      # one tile in the most shares
    ([700, 3, 260], [0, 40, 900], 8, 1, 64),
    ([1000], [0], 16, 16, 64)])
def test_prompt_layouts(lens, held, heads, kv_heads, d):
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 64)
    cache = make_cache(kv_heads, 64, d, n_pages, table, seed=3)
    batch, cu = batch_of(lens, held)
    q = randn(8, sum(lens), heads, d).bfloat16()
    out = torch.full_like(q, float("nan"))
    scd.scd_cache_attend(cache, batch, q, out)
    assert bool(torch.isfinite(out).all())
    rows = sorted({0, 31, 32, 63, 64, 65, 127, 128, sum(lens) // 2, sum(lens) - 2, sum(lens) - 1} & set(range(sum(lens))))
    sampled(cache, table, cu, held, q, out, rows)


def test_many_requests_of_prompt_size():
    """More requests than a workgroup of the prompts' kernel looks through at once, some of them empty."""
    rng = np.random.default_rng(5)
    lens = (rng.integers(0, 80, 700) * (rng.random(700) < 0.9)).tolist()
    held = rng.integers(0, 100, 700).tolist()
    table, n_pages = table_of(rng, lens, held, 16)
    cache = make_cache(1, 16, 64, n_pages, table, seed=3)
    batch, cu = batch_of(lens, held)
    q = randn(8, sum(lens), 4, 64).bfloat16()
    out = torch.full_like(q, float("nan"))
    scd.scd_cache_attend(cache, batch, q, out)
    assert bool(torch.isfinite(out).all())
    sampled(cache, table, cu, held, q, out, rng.integers(0, sum(lens), 60).tolist() + [0, sum(lens) - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held", [
    ([1], [510]), ([1], [511]), ([1], [512]), ([1], [4095]), ([1, 1, 1, 1], [2000, 0, 513, 127]),
    ([1, 0, 2, 1, 0], [9000, 5, 31, 640, 0]), ([3] * 40, list(range(0, 1200, 30)))])
def test_whole_and_cut_segments(dtype, lens, held):
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 32)
    cache = make_cache(2, 32, 64, n_pages, table, seed=3)
    check_attend(cache, lens, held, table, randn(8, sum(lens), 6, 64).to(DT[dtype]), dtype)


def test_one_workspace_for_calls_of_every_shape():
    """One buffer, zero before its first use, serves cut segments and prompts in turn and is left ready."""
    shapes = [([1, 1], [3000, 100]), ([300], [2000]), ([1] * 20, [700] * 20), ([2, 1], [9000, 4])]
    worlds = []
    for lens, held in shapes:
        table, n_pages = table_of(np.random.default_rng(4), lens, held, 64)
        cache = make_cache(2, 64, 128, n_pages, table, seed=3)
        batch, _ = batch_of(lens, held)
        q = randn(8, sum(lens), 8, 128).bfloat16()
        alone = torch.empty_like(q)
        scd.scd_cache_attend(cache, batch, q, alone)
        worlds.append((cache, batch, q, alone, torch.empty_like(q)))
    nbytes = max(scd.scd_cache_attend_workspace_bytes(c, b, 8) for c, b, *_ in worlds)
    workspace = torch.full((nbytes,), 0xAB, dtype=torch.uint8, device="cuda")
    workspace[:2048] = 0  # SCD_ATTEND_COUNTER_BYTES; the rest may hold anything
    for _ in range(3):
        for cache, batch, q, alone, out in worlds:
            scd.scd_cache_attend(cache, batch, q, out, workspace=workspace)
            assert torch.equal(out, alone)
            assert not bool(workspace[:2048].any())
    short = workspace[:nbytes - 16]
    with pytest.raises(scd.ScdError, match="workspace_bytes"):
        for cache, batch, q, _, out in worlds:
            scd.scd_cache_attend(cache, batch, q, out, workspace=short)


def test_captured_attention_grows_into_cut_segments():
    """A step captured while segments are whole, replayed until they are cut over many workgroups."""
    n, heads, kv_heads, d, size = 2, 8, 2, 128, 64
    start, longest = [40, 250], 6000
    rng = np.random.default_rng(6)
    table = rng.permutation(2 * (longest // size + 1)).reshape(2, -1)
    cache = make_cache(kv_heads, size, d, table.size, table, seed=9)
    q, pos0 = randn(1, n, heads, d).bfloat16(), ints(start)
    batch = scd.Batch(n, ints([0, 1, 2]), pos0)
    out = torch.empty_like(q)
    call = scd.prepare_cache_attend(cache, batch, q, out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    eager = torch.empty_like(out)
    for grow in (0, 1, 300, 900, 3000, 5600, 2):
        pos0.copy_(ints([s + grow for s in start]))
        graph.replay()
        scd.scd_cache_attend(cache, batch, q, eager)
        assert torch.equal(out, eager)
        check_attend(cache, [1, 1], [s + grow for s in start], table, q, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held", [
    ([2] * 16, [590 + i for i in range(16)]),           # 128 segments of 5 steps: whole
    ([4] * 16, [100 * i for i in range(16)]),           # ragged, up to 13 steps: whole
    ([1] * 40 + [2], [20 + i for i in range(40)] + [9000]),  # one long among short ones: cut, into many parts
    ([1] * 70, [120] * 69 + [700]),                     # segments of one step, the longest 6: whole
    ([0, 3, 0, 0], [9, 4000, 7, 8000])])                # the longest has no new token
def test_uneven_requests_whole_and_cut(dtype, lens, held):
    """Both sides of the rule between whole segments and equal shares, uneven requests among them."""
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 32)
    cache = make_cache(4, 32, 64, n_pages, table, seed=3)
    q = (randn(8, sum(lens), 16, 64) * 2).to(DT[dtype])
    check_attend(cache, lens, held, table, q, dtype)


@pytest.mark.parametrize("lens,held", [([8, 7], [0, 3]), ([8, 8], [5, 60]), ([1] * 7 + [60], [0] * 8), ([700], [33])])
@pytest.mark.parametrize("heads", [1, 3, 8])
def test_append_few_and_many_rows(lens, held, heads):
    """Both sides of the rule between a wave a head and a workgroup a page, one and several heads a workgroup."""
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 64)
    cache = make_cache(heads, 64, 128, n_pages, table)
    batch, cu = batch_of(lens, held)
    k, v = (randn(s, sum(lens), heads, 128).bfloat16() for s in (1, 2))
    turns = scd.scd_rotary_table(scd.Rotary(128, 5e5), 1000)
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v, turns)
    kx = O.rotate(f64(k), positions(lens, held), O.frequencies(128, 5e5))
    check_append(cache, before, table, cu, held, (kx, f64(v)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held,size", [([32, 31], [0, 50], 64), ([32, 32], [5, 60], 64), ([31], [17], 16),
                                            ([140, 1, 1, 1, 1], [9, 0, 63, 64, 3], 64), ([150], [5], 128)])
def test_append_on_both_sides_of_32_rows_a_request(dtype, lens, held, size):
    table, n_pages = table_of(np.random.default_rng(5), lens, held, size)
    cache = make_cache(3, size, 128, n_pages, table)
    batch, cu = batch_of(lens, held)
    k, v = (randn(s, sum(lens), 3, 128).to(DT[dtype]) for s in (1, 2))
    turns = scd.scd_rotary_table(scd.Rotary(128, 5e5), 1000)
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v, turns)
    kx = O.rotate(f64(k), positions(lens, held), O.frequencies(128, 5e5))
    check_append(cache, before, table, cu, held, (kx, f64(v)))


def test_append_of_a_long_batch_reads_back():
    """Enough pages that a workgroup takes several heads of both branches, ragged, against the append of every
    request alone."""
    lens, held = [3001, 64, 1, 5000], [0, 10, 0, 77]
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 32)
    cache, alone = (make_cache(8, 32, 64, n_pages, table, seed=3) for _ in range(2))
    batch, cu = batch_of(lens, held)
    k, v = (randn(s, sum(lens), 8, 64).bfloat16() for s in (1, 2))
    turns = scd.scd_rotary_table(scd.Rotary(64, 1e4, layout="interleaved"), 6000)
    scd.scd_cache_append(cache, batch, k, v, turns)
    for b, (n, h) in enumerate(zip(lens, held)):
        one = scd.PagedCache(alone.k_pages, alone.v_pages, alone.k_scales, alone.v_scales, alone.page_table[b:b + 1].contiguous())
        scd.scd_cache_append(one, scd.Batch(n, None, ints([h])), k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]], turns)
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        assert torch.equal(getattr(cache, name), getattr(alone, name)), name
