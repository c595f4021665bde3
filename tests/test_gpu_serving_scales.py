"""Attention over pages whose value scales lie far apart, in both kernels: what a position weighs in the softmax does
not depend on its page's value scale, and no scale reaches rows that do not see its page."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from tests.test_gpu_serving import DT, EPS, _gpu, batch_of, f64, ints, make_cache, randn, table_of  # noqa: F401

pytestmark = pytest.mark.gpu


def reference(cache, table, lens, held, q, scale, rows=None):
    """In fp64, for the given packed rows (None: all): out, sum_j p_j |v_j|, scale * max_j sum |q||k_j|, and
    max_j p_j * (value scale of j) times the positions seen."""
    size, heads, d = cache.k_pages.shape[2], cache.n_kv_heads, cache.head_dim
    n_pages, group = cache.k_pages.shape[0], q.shape[1] // heads
    rows = range(q.shape[0]) if rows is None else rows
    bytes_ = [p.cpu().numpy().astype(np.float64) for p in (cache.k_pages, cache.v_pages)]
    ks, vs = f64(cache.k_scales), f64(cache.v_scales)
    cu = np.concatenate([[0], np.cumsum(lens)])
    q = f64(q)
    shape = (len(rows), heads * group, d)
    out, mass, reach, peak = np.zeros(shape), np.zeros(shape), np.zeros(shape[:2]), np.zeros(shape[:2])
    gathered = {}
    for i, t in enumerate(rows):
        b = int(np.searchsorted(cu, t, side="right")) - 1
        if b not in gathered:
            pos = np.arange(held[b] + lens[b])
            ids = np.array([table[b, c] if c < table.shape[1] else -1 for c in pos // size])
            pos = pos[(ids >= 0) & (ids < n_pages)]
            ids = ids[(ids >= 0) & (ids < n_pages)]
            wide = [(x[ids, :, pos % size] * s[ids][:, :, None]).transpose(1, 0, 2) for x, s in zip(bytes_, (ks, vs))]
            gathered[b] = pos, wide, vs[ids].T
        pos, (k, v), each = gathered[b]
        m = int(np.searchsorted(pos, held[b] + t - cu[b], side="right"))
        if m == 0:
            continue
        for h in range(heads * group):
            g = h // group
            s = scale * (k[g, :m] @ q[t, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mass[i, h] = p @ v[g, :m], p @ np.abs(v[g, :m])
            reach[i, h] = abs(scale) * (np.abs(k[g, :m]) @ np.abs(q[t, h])).max()
            peak[i, h] = (p * each[g, :m]).max() * m
    return out, mass, reach, peak


def check(cache, table, lens, held, q, dtype, scale=None, rows=None, prompt=False):
    batch, _ = batch_of(lens, held)
    out = torch.full_like(q, float("nan"))
    scd.scd_cache_attend(cache, batch, q, out, scale)
    scale = cache.head_dim ** -0.5 if scale is None else scale
    want, mass, reach, peak = reference(cache, table, lens, held, q, scale, rows)
    # Scores are off by at most 2^-19 of scale * sum |q||k|, their weights by twice that and the exponential's own 2^-18;
    # bf16 calls' weights carry 11 bits.  The prompts' are fp16 with 2^11 for the heaviest position (weight times value
    # scale): a lighter one is off by 2^-25 of that unit at most, times a value of at most 127: 2^-29 of the peak.
    rel = 2 * 2.0 ** -19 * reach[..., None] + 2.0 ** -18 + (2.0 ** -10 if dtype == "bf16" else 0.0)
    bound = rel * mass + 0.51 * EPS[dtype] * np.abs(want) + (2.0 ** -29 * peak[..., None] if prompt else 0.0)
    got = f64(out if rows is None else out[list(rows)])
    assert np.all(np.abs(got - want) <= bound + 2.0 ** -133), float(np.nanmax(np.abs(got - want) / (bound + 2.0 ** -133)))
    return out


# 8 query heads over 2: 90 and 80 tokens are 340 rows a request, which the prompts' kernel takes in bf16 from 64
# channels on; one share of their tiles where the table holds at most 256 positions, two otherwise.
SHAPES = [("bf16", 64, [1, 1], [300, 77]), ("f32", 64, [1, 1], [300, 77]), ("f32", 128, [40, 3], [100, 40]),
          ("bf16", 32, [90, 80], [100, 40]), ("bf16", 64, [90, 80], [100, 40]), ("bf16", 128, [90, 80], [100, 40]),
          ("bf16", 64, [90, 80], [300, 77]), ("bf16", 128, [90, 80], [300, 77])]


def world(dtype, d, lens, held, size=16):
    table, n_pages = table_of(np.random.default_rng(4), lens, held, size)
    cache = make_cache(2, size, d, n_pages, table, seed=3)
    return cache, table, randn(8, sum(lens), 8, d).to(DT[dtype]), dtype == "bf16" and d >= 64 and sum(lens) > 64


@pytest.mark.parametrize("dtype,d,lens,held", SHAPES)
@pytest.mark.parametrize("quiet", [1e-3, 1e-6, 1e-8, 1e-9, 1e-10, 1e-20, 1e-32, 0.0])
def test_quiet_pages_count_in_the_softmax(dtype, d, lens, held, quiet):
    """Every other page's values are `quiet` of the rest's; with 0 they are zeros, as the append stores them."""
    cache, table, q, prompt = world(dtype, d, lens, held)
    for b in range(2):
        ids = ints(table[b, 1::2]).long()
        cache.v_scales[ids] *= quiet
        if quiet == 0.0:
            cache.v_pages[ids] = 0
    check(cache, table, lens, held, q, dtype, prompt=prompt)


@pytest.mark.parametrize("dtype,d,lens,held", SHAPES)
@pytest.mark.parametrize("scale", [None, -0.3])
def test_wide_ranges(dtype, d, lens, held, scale):
    """Scores of hundreds, scales from 1e-30 to 1e4 and zeros side by side, queries of very different size, a negative
    softmax scale."""
    cache, table, q, prompt = world(dtype, d, lens, held)
    cache.v_scales[table[0, 3]] = 1e4
    cache.v_scales[table[0, 5]] = 1e-30
    cache.v_scales[table[1, 0]] = 1e-30
    cache.v_scales[table[1, 2]] = 1e-9
    cache.v_scales[table[0, 0]] = 0.0
    cache.v_pages[table[0, 0]] = 0
    cache.k_scales[table[0, 2]] = 0.0
    cache.k_pages[table[0, 2]] = 0
    q = (q.float() * torch.logspace(-6, 1, sum(lens), device="cuda").view(-1, 1, 1)).to(DT[dtype])
    check(cache, table, lens, held, q, dtype, scale, prompt=prompt)


@pytest.mark.parametrize("dtype,d,lens,held", SHAPES)
@pytest.mark.parametrize("loud", [1e6, 1e15, 1e25, 1e35])
def test_pages_of_zeros_beside_loud_ones(dtype, d, lens, held, loud):
    cache, table, q, prompt = world(dtype, d, lens, held)
    for b in range(2):
        cache.v_scales[ints(table[b, 0::3]).long()] *= loud
        ids = ints(table[b, 1::3]).long()
        cache.v_scales[ids] = 0.0
        cache.v_pages[ids] = 0
    check(cache, table, lens, held, q, dtype, prompt=prompt)


@pytest.mark.parametrize("dtype,d,lens,held", SHAPES)
@pytest.mark.parametrize("power", [-118, -110, -100, 60, 110])
def test_scales_near_the_ends_of_their_range(dtype, d, lens, held, power):
    """All values of about 2^power: their scales have no ordinary page beside them."""
    cache, table, q, prompt = world(dtype, d, lens, held)
    cache.v_scales.mul_(2.0 ** (power // 2)).mul_(2.0 ** (power - power // 2))
    check(cache, table, lens, held, q, dtype, prompt=prompt)


@pytest.mark.parametrize("dtype,tokens,kv_heads,heads,zeros,ordinary", [
    ("bf16", 2048, 8, 32, 19000, 2500),    # prompts, no shares: a workgroup goes over all positions
    ("bf16", 64, 1, 8, 600000, 1500),      # prompts in 64 shares
    ("bf16", 1, 8, 32, 40000, 100), ("f32", 1, 2, 2, 300000, 77)])
def test_many_positions_of_zeros(dtype, tokens, kv_heads, heads, zeros, ordinary):
    """A long run of pages of zeros (scale 0) in front of ordinary ones; scores rise by just under 4 log2 units after the
    first 64 positions, so that every position weighs 15 times what the first ones do."""
    size, d, total = 64, 64, zeros // 64 * 64 + ordinary
    n_pages = -(-total // size)
    table = np.random.default_rng(2).permutation(n_pages)[None]
    cache = make_cache(kv_heads, size, d, n_pages, table, seed=3)
    cache.k_pages.zero_()
    cache.k_pages[..., 0] = 1
    cache.k_pages[int(table[0, 0]), :, :, 0] = 0
    cache.k_scales.fill_(3.9 * float(np.log(2.0)))
    ids = ints(table[0, :zeros // size]).long()
    cache.v_pages[ids] = 0
    cache.v_scales[ids] = 0.0
    q = randn(8, tokens, heads, d).to(DT[dtype])
    q[..., 0] = 1.0
    rows = sorted({0, tokens // 3, tokens - 1})
    check(cache, table, [tokens], [total - tokens], q, dtype, scale=1.0, rows=rows, prompt=tokens > 1)


@pytest.mark.parametrize("dtype,tokens,kv_heads,heads", [("bf16", 2048, 8, 32), ("bf16", 1, 8, 32), ("f32", 3, 2, 8)])
@pytest.mark.parametrize("gains", [(1.0, 1e18, 1.0), (1e18, 1.0, 0.0), (0.0, 1.0, 1e-18), (1.0, 0.0, 1.0), (1e18, 1.0, 1e18)])
def test_long_runs_of_pages_far_apart(dtype, tokens, kv_heads, heads, gains):
    """Value scales that change every 16384 positions, as many as a workgroup of the prompts' kernel lists at once; the
    parts that a few rows' positions are cut into have pages of one kind and of two."""
    size, d, run = 64, 64, 16384
    total = 3 * run - 1000
    n_pages = -(-total // size)
    table = np.random.default_rng(2).permutation(n_pages)[None]
    cache = make_cache(kv_heads, size, d, n_pages, table, seed=3)
    for i, gain in enumerate(gains):
        ids = ints(table[0, i * run // size:(i + 1) * run // size]).long()
        cache.v_scales[ids] *= gain
        if gain == 0.0:
            cache.v_pages[ids] = 0
    q = randn(8, tokens, heads, d).to(DT[dtype])
    rows = sorted({0, tokens // 3, tokens - 1})
    check(cache, table, [tokens], [total - tokens], q, dtype, rows=rows, prompt=tokens > 1)


@pytest.mark.parametrize("dtype,lens,held", [("bf16", [90, 80, 100], [100, 64, 3]), ("bf16", [90, 80, 100], [400, 64, 3]),
                                             ("bf16", [5, 40, 1], [100, 96, 3]), ("f32", [90, 80, 100], [100, 64, 3])])
def test_nan_stays_with_the_rows_that_see_it(dtype, lens, held):
    """A query that is not a number; key and value scales that are not, of pages that all rows of a request reach and
    of pages that its later rows reach."""
    cache, table, q, prompt = world(dtype, 64, lens, held)
    batch, cu = batch_of(lens, held)
    sound = check(cache, table, lens, held, q, dtype, prompt=prompt)
    late = held[1] + lens[1] // 2  # a position whose page the earlier rows of request 1 do not see
    cache.k_scales[table[1, late // 16], 0] = float("nan")
    cache.v_scales[table[1, late // 16], 1] = float("nan")
    cache.v_scales[table[2, 0], 1] = float("nan")
    q[0, 1, 5] = float("nan")
    out = torch.full_like(q, float("inf"))
    scd.scd_cache_attend(cache, batch, q, out)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[0, 1] = True
    first = late // 16 * 16 - held[1]  # the first row that reaches the page
    assert 0 < first < lens[1]
    want[cu[1] + first:cu[2]] = True
    want[cu[2]:, 4:] = True
    assert torch.equal(torch.isnan(out), want)
    # a prompt's weights may be taken against another running maximum: 11 bits each way
    x, y = out[~want].double(), sound[~want].double()
    assert float((x - y).abs().max()) <= 2.0 ** -9 * float(y.abs().max())
