"""Rotary positions, the paged 8-bit cache and attention over it, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import serving_oracle as O

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = {"bf16": 2.0 ** -7, "f32": 2.0 ** -23}  # spacing of the output type; one rounding is half of it


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


def f64(t):
    return t.double().cpu().numpy()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def batch_of(lens, held):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()
    return scd.Batch(sum(lens), ints(cu), ints(held)), cu


def positions(lens, held):
    return [h + i for n, h in zip(lens, held) for i in range(n)]


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def strided(x, how):
    """x's values behind other strides."""
    t, h, d = x.shape
    if how == "dense":
        return x.clone()
    if how == "fused":     # heads of a wider row
        y = torch.zeros(t, h + 3, d, dtype=x.dtype, device=x.device)[:, 2:2 + h]
    elif how == "heads_first":
        y = torch.zeros(h, t, d, dtype=x.dtype, device=x.device).transpose(0, 1)
    elif how == "odd":     # rows that start on an element only
        y = torch.zeros(t * h * (d + 1) + 1, dtype=x.dtype, device=x.device)[1:].view(t, h, d + 1)[..., :d]
    y.copy_(x)
    return y


# ---- rotary ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("scaling,kw", [
    ("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
    ("by_parts", dict(factor=8.0, low=1.0, high=4.0, trained_positions=8192)),
    ("by_parts", dict(factor=16.0, trained_positions=4096, attention_factor=1.2773)),
    ("given", dict(frequencies=[0.5 ** i for i in range(16)]))])
def test_rotary_table(scaling, kw):
    r = scd.Rotary(64, 5e5, rotary_dim=32, scaling=scaling, **kw)
    got = scd.scd_rotary_table(r, 40001).buffer.view(torch.float32).view(40001, 16, 2)
    given = kw.get("frequencies")
    w = np.array(given) if given else O.frequencies(32, 5e5, scaling, kw.get("factor", 1.0), kw.get("low", 1.0),
                                                    kw.get("high", 32.0), kw.get("trained_positions", 0))
    gain = kw.get("attention_factor", 1.0)
    angle = np.arange(40001)[:, None] * w
    for i, want in enumerate((gain * np.cos(angle), gain * np.sin(angle))):
        # one rounding to fp32, and fp64 angles of up to 4e4 that may be an ulp apart
        assert np.all(np.abs(f64(got[..., i]) - want) <= 2.0 ** -24 * np.abs(want) + 4e4 * 2.0 ** -51)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("head_dim,rotary_dim,how", [
    (128, 128, "dense"), (128, 64, "fused"), (64, 64, "heads_first"), (64, 16, "odd"), (32, 32, "fused"),
    (80, 32, "dense"), (80, 20, "dense"), (96, 96, "fused"), (10, 6, "dense"), (6, 2, "odd"), (256, 256, "dense"),
    (512, 48, "dense")])
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary(dtype, layout, head_dim, rotary_dim, how, transpose):
    lens, held = [3, 0, 1, 70, 0], [0, 5, 4000, 17, 2]
    batch, cu = batch_of(lens, held)
    pos = positions(lens, held)
    table = scd.scd_rotary_table(scd.Rotary(head_dim, 1e4, rotary_dim=rotary_dim, layout=layout,
                                            attention_factor=1.25), 4001)
    q, k = (strided(randn(s, sum(lens), h, head_dim).to(DT[dtype]), how) for s, h in ((1, 5), (2, 3)))
    w = O.frequencies(rotary_dim, 1e4)
    for keys in (True, False):
        outs = [strided(torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda"), how) for x in (q, k)]
        scd.scd_rotary(table, batch, q, k if keys else None, outs[0], outs[1] if keys else None, transpose)
        for x, y in list(zip((q, k), outs))[:2 if keys else 1]:
            want = O.rotate(f64(x), pos, w, layout, 1.25, transpose)
            # fp32: two products and a sum of factors rounded once (4 roundings of at most 1.25 * sqrt(2)
            # times the pair); then one rounding to the output's type
            amp = 1.25 * 1.5 * np.abs(f64(x)).max()
            assert np.all(np.abs(f64(y) - want) <= 0.51 * EPS[dtype] * np.abs(want) + 4 * 2.0 ** -24 * amp)
            assert torch.equal(y[..., rotary_dim:], x[..., rotary_dim:])
    place = [q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)]
    scd.scd_rotary(table, batch, *place, *place, transpose)
    scd.scd_rotary(table, batch, q, k, *outs, transpose)
    assert torch.equal(place[0], outs[0]) and torch.equal(place[1], outs[1])


@pytest.mark.parametrize("tokens,heads,kv_heads", [(1, 32, 8), (5000, 32, 8), (4999, 64, 8), (7, 8, 8), (3001, 1, 1)])
def test_rotary_many_rows(tokens, heads, kv_heads):
    """Every row of batches of all sizes, against the fp64 rotation by complex numbers."""
    split = [tokens // 3, tokens - tokens // 3]
    batch, _ = batch_of(split, [11, 0])
    pos = torch.tensor(positions(split, [11, 0]), dtype=torch.float64)
    r = scd.Rotary(128, 5e5)
    table = scd.scd_rotary_table(r, 6000)
    q, k = randn(3, tokens, heads, 128).bfloat16(), randn(4, tokens, kv_heads, 128).bfloat16()
    out = torch.empty_like(q), torch.empty_like(k)
    scd.scd_rotary(table, batch, q, k, *out)
    turn = torch.polar(torch.ones(1, dtype=torch.float64), pos[:, None] * torch.from_numpy(O.frequencies(128, 5e5)))[:, None]
    for x, y in zip((q, k), out):
        x = x.double().cpu()
        z = torch.complex(x[..., :64], x[..., 64:]) * turn
        want = torch.cat([z.real, z.imag], -1)
        assert bool(((y.double().cpu() - want).abs() <= 0.51 * EPS["bf16"] * want.abs() + 1e-5).all())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient_against_differences(layout):
    """f(x) = <g, R x> (R linear): its gradient is the transposed call on g, its differences exact."""
    batch, _ = batch_of([4, 2], [3, 900])
    table = scd.scd_rotary_table(scd.Rotary(32, 1e4, rotary_dim=16, layout=layout, attention_factor=1.1), 1000)
    x, g = randn(5, 6, 2, 32), randn(6, 6, 2, 32)
    y, grad = torch.empty_like(x), torch.empty_like(x)
    scd.scd_rotary(table, batch, g, None, grad, None, transpose=True)

    def f(x):
        scd.scd_rotary(table, batch, x, None, y, None)
        return float((g.double() * y.double()).sum())

    for t, h, c in [(0, 0, 0), (3, 1, 9), (4, 0, 5), (5, 1, 15), (5, 0, 31)]:
        e = torch.zeros_like(x)
        e[t, h, c] = 0.5
        # each f sums 384 products of rounded values of about 1.1: 2^-23 * 384 is above their error
        assert abs((f(x + e) - f(x - e)) - float(grad[t, h, c])) <= 2.0 ** -23 * 384 * 4


# ---- the paged cache -------------------------------------------------------------------------------
def make_cache(heads, size, d, n_pages, table, seed=0, fill=True):
    """A pool with arbitrary bytes and, in pages not yet begun, scales that are not numbers."""
    gen = torch.Generator().manual_seed(seed)
    pages = [torch.randint(-127, 128, (n_pages, heads, size, d), generator=gen, dtype=torch.int8).cuda() for _ in "kv"]
    scales = [(0.01 + torch.rand(n_pages, heads, generator=gen) * 0.03).cuda() if fill else
              torch.full((n_pages, heads), float("nan"), device="cuda") for _ in "kv"]
    return scd.PagedCache(*pages, *scales, ints(table))


def table_of(rng, lens, held, size, extra=2):
    """Distinct pages in scattered order; unused columns name a page that nothing else does."""
    need = [-(-(n + h) // size) for n, h in zip(lens, held)]
    order = rng.permutation(sum(need)) + 1
    table = np.zeros((len(lens), max(need) + extra), dtype=np.int64)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + 2


def check_append(cache, before, table, cu, pos0, rows):
    """The cache after an append against the oracle: scales within their roundings, bytes equal but
    where the value lies within 1e-4 of a tie (x / scale carries a few 2^-24 of at most 127)."""
    for (pages, scales), (old_pages, old_scales), x in zip(
            ((cache.k_pages, cache.k_scales), (cache.v_pages, cache.v_scales)), before, rows):
        want, want_scale = old_pages.astype(np.float64), old_scales.astype(np.float64)
        ratio = O.append(want, want_scale, table, cu, pos0, x)
        got, got_scale = f64(pages), f64(scales)
        assert np.array_equal(np.isnan(got_scale), np.isnan(want_scale))
        sound = ~np.isnan(want_scale)
        assert np.all(np.abs(got_scale - want_scale)[sound] <= 4 * 2.0 ** -24 * want_scale[sound])
        off = (got != want) & sound[:, :, None, None]
        near = np.abs(np.abs(ratio - np.floor(ratio)) - 0.5) < 1e-4
        assert np.all(~off | (near & (np.abs(got - want) <= 1)))


def state(cache):
    return [(p.cpu().numpy().copy(), s.cpu().numpy().copy())
            for p, s in ((cache.k_pages, cache.k_scales), (cache.v_pages, cache.v_scales))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,size", [(128, 64), (128, 128), (128, 16), (64, 16), (64, 128), (32, 16), (32, 32), (32, 128)])
@pytest.mark.parametrize("lens,held", [
    ([1], [0]), ([1, 1, 0, 1, 1], [15, 16, 9, 127, 300]), ([37, 0, 200, 1, 5], [0, 4, 77, 63, 250])])
@pytest.mark.parametrize("turn,how", [(None, "dense"), (("half", 1.0), "fused"), (("interleaved", 0.5), "odd")])
def test_append(dtype, d, size, lens, held, turn, how):
    rng = np.random.default_rng(7)
    table, n_pages = table_of(rng, lens, held, size)
    cache = make_cache(3, size, d, n_pages, table)
    batch, cu = batch_of(lens, held)
    k, v = (strided((randn(s, sum(lens), 3, d) * a).to(DT[dtype]), how) for s, a in ((1, 1.0), (2, 3.0)))
    rot, kx = None, f64(k)
    if turn is not None:
        rd = int(d * turn[1])
        rot = scd.scd_rotary_table(scd.Rotary(d, 1e4, rotary_dim=rd, layout=turn[0]), 600)
        kx = O.rotate(kx, positions(lens, held), O.frequencies(rd, 1e4), turn[0])
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v, rot)
    check_append(cache, before, table, cu, held, (kx, f64(v)))


@pytest.mark.parametrize("rotary_dim,layout", [(20, "half"), (20, "interleaved"), (2, "half"), (8, "half")])
def test_append_odd_rotary_dims(rotary_dim, layout):
    lens, held = [40, 3], [5, 0]
    table, n_pages = table_of(np.random.default_rng(3), lens, held, 16)
    cache = make_cache(2, 16, 64, n_pages, table)
    batch, cu = batch_of(lens, held)
    k, v = randn(1, 43, 2, 64), randn(2, 43, 2, 64)
    rot = scd.scd_rotary_table(scd.Rotary(64, 1e4, rotary_dim=rotary_dim, layout=layout), 64)
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v, rot)
    kx = O.rotate(f64(k), positions(lens, held), O.frequencies(rotary_dim, 1e4), layout)
    check_append(cache, before, table, cu, held, (kx, f64(v)))


def test_append_one_token_at_a_time_grows_scales():
    """70 tokens, each louder than the last now and then: earlier values move to the grown scale."""
    table, n_pages = table_of(np.random.default_rng(1), [70, 70], [0, 0], 32)
    cache = make_cache(2, 32, 64, n_pages, table, fill=False)
    k, v = (randn(s, 70, 2, 2, 64) * torch.linspace(0.1, 2.0, 70, device="cuda").view(-1, 1, 1, 1) for s in (1, 2))
    for i in range(70):
        batch, cu = batch_of([1, 1], [i, i])
        before = state(cache)
        scd.scd_cache_append(cache, batch, k[i], v[i])
        check_append(cache, before, table, cu, [i, i], (f64(k[i]), f64(v[i])))
    out = [torch.empty(140, 2, 64, device="cuda") for _ in "kv"]
    scd.scd_cache_read(cache, scd.Batch(140, ints([0, 70, 140])), *out)
    for x, y, scales in ((k, out[0], cache.k_scales), (v, out[1], cache.v_scales)):
        want = x.transpose(0, 1).reshape(140, 2, 64)
        # half a step, and up to ten growths of half a step of a smaller scale each
        assert float((y - want).abs().max()) <= 6 * float(scales[ints(table[:, :3]).long().flatten()].max())


def test_append_zeros_small_values_and_non_finite_values():
    table, n_pages = table_of(np.random.default_rng(1), [8, 8, 8, 8, 8], [0, 3, 0, 3, 0], 16)
    cache = make_cache(2, 16, 32, n_pages, table)
    batch, cu = batch_of([8] * 5, [0, 3, 0, 3, 0])
    k, v = randn(1, 40, 2, 32), randn(2, 40, 2, 32)
    k[0:8] = 0.0
    k[8:16] = 0.0          # behind three held rows: their scale stays
    k[16:24] *= 1e-38 / 5  # below the smallest scale
    k[27, 1, 3] = float("nan")
    v[33, 0, 31] = float("inf")
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v)
    check_append(cache, before, table, cu, [0, 3, 0, 3, 0], (f64(k), f64(v)))
    assert float(cache.k_scales[table[0, 0]].max()) == 0.0
    out = [torch.empty(11 * 5, 2, 32, device="cuda") for _ in "kv"]
    scd.scd_cache_read(cache, scd.Batch(55, ints([0, 11, 22, 33, 44, 55])), *out)
    bad = torch.isnan(out[0])
    assert bool(bad[33:44, 1].all()) and not bool(bad[33:44, 0].any()) and not bool(bad[:33].any())
    assert bool(torch.isnan(out[1][44:52, 0]).all()) and not bool(torch.isnan(out[1][44:52, 1]).any())
    # the page begun again is sound
    batch, cu = batch_of([2, 0, 0, 2, 2], [0] * 5)
    scd.scd_cache_append(cache, batch, randn(5, 6, 2, 32), randn(6, 6, 2, 32))
    assert bool(torch.isfinite(cache.k_scales[table[3, 0]]).all())
    assert bool(torch.isfinite(cache.v_scales[table[4, 0]]).all())


def test_holes_and_positions_outside_the_table():
    """Rows at holes, past the table and at negative positions: dropped, read as zeros."""
    table = np.array([[1, -1, 2, 99], [3, 4, 5, 6]])
    cache = make_cache(2, 16, 64, 8, table)
    lens, held = [60, 30], [3, 50]
    batch, cu = batch_of(lens, held)
    k, v = randn(1, 90, 2, 64), randn(2, 90, 2, 64)
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v)
    check_append(cache, before, table, cu, held, (f64(k), f64(v)))
    out = [torch.full((90, 2, 64), float("nan"), device="cuda") for _ in "kv"]
    scd.scd_cache_read(cache, batch, *out)
    for y in out:
        pos = np.array(positions(lens, held))
        none = torch.tensor([O.page_of(table, 8, 16, 0 if t < 60 else 1, p) < 0 for t, p in enumerate(pos)])
        assert bool((y[none.cuda()] == 0).all()) and bool((y[~none.cuda()] != 0).any(2).any(1).all())
    before = state(cache)
    batch, cu = batch_of([5, 3], [-2, -7])
    scd.scd_cache_append(cache, batch, k[:8], v[:8])
    check_append(cache, before, table, cu, [-2, -7], (f64(k[:8]), f64(v[:8])))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,size,how", [(128, 64, "dense"), (64, 16, "odd"), (32, 128, "heads_first"), (128, 32, "fused")])
def test_read(dtype, d, size, how):
    lens, first = [0, 77, 1, 130], [0, 5, 0, 40]
    table, n_pages = table_of(np.random.default_rng(2), lens, first, size)
    cache = make_cache(3, size, d, n_pages, table)
    batch, _ = batch_of(lens, first)
    out = [strided(torch.full((208, 3, d), float("nan"), dtype=DT[dtype], device="cuda"), how) for _ in "kv"]
    scd.scd_cache_read(cache, batch, *out)
    req = sum([[b] * n for b, n in enumerate(lens)], [])
    pos = np.array(positions(lens, first))
    page, slot = torch.from_numpy(table[req, pos // size]).cuda(), torch.from_numpy(pos % size).cuda()
    for y, pages, scales in zip(out, (cache.k_pages, cache.v_pages), (cache.k_scales, cache.v_scales)):
        assert torch.equal(y, (pages[page, :, slot].float() * scales[page][:, :, None]).to(DT[dtype]))


# ---- attention -------------------------------------------------------------------------------------
def check_attend(cache, lens, held, table, q, dtype, scale=None, how="dense"):
    batch, cu = batch_of(lens, held)
    d = cache.head_dim
    out = strided(torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda"), how)
    scd.scd_cache_attend(cache, batch, strided(q, how), out, scale)
    scale = d ** -0.5 if scale is None else scale
    want, mass, reach = O.attend(f64(q), cache.k_pages.cpu().numpy(), cache.v_pages.cpu().numpy(),
                                 cache.k_scales.cpu().numpy(), cache.v_scales.cpu().numpy(), table, cu, held, scale)
    # A score is off by at most 2^-19 of scale * sum |q||k| (fp32 sums of up to 128 products), its
    # weight by twice that and the exponential's own 2^-18; bf16 weights carry 11 bits or more.
    rel = 2 * 2.0 ** -19 * reach[..., None] + 2.0 ** -18 + (2.0 ** -10 if dtype == "bf16" else 0.0)
    err = np.abs(f64(out) - want)
    assert np.all(err <= rel * mass + 0.51 * EPS[dtype] * np.abs(want)), float((err / (rel * mass + 1e-30)).max())
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,size,heads,kv_heads", [
    (128, 64, 8, 2), (128, 16, 7, 1), (64, 16, 4, 4), (64, 128, 8, 1), (32, 32, 6, 2), (128, 32, 34, 2), (32, 128, 40, 1)])
@pytest.mark.parametrize("lens,held", [
    ([1], [0]), ([1, 1, 0, 1, 1, 1], [31, 32, 9, 0, 500, 130]), ([5, 0, 3, 2, 1], [0, 4, 77, 640, 16]),
    ([100], [0]), ([129, 1, 70], [0, 300, 45])])
def test_attend(dtype, d, size, heads, kv_heads, lens, held):
    table, n_pages = table_of(np.random.default_rng(4), lens, held, size)
    cache = make_cache(kv_heads, size, d, n_pages, table, seed=3)
    q = (randn(8, sum(lens), heads, d) * 2).to(DT[dtype])
    check_attend(cache, lens, held, table, q, dtype)


@pytest.mark.parametrize("how", ["fused", "heads_first", "odd"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_strides(dtype, how):
    for lens, held in (([1, 1, 1], [40, 5, 77]), ([90, 1], [10, 3])):
        table, n_pages = table_of(np.random.default_rng(4), lens, held, 16)
        cache = make_cache(2, 16, 64, n_pages, table, seed=3)
        check_attend(cache, lens, held, table, randn(8, sum(lens), 6, 64).to(DT[dtype]), dtype, how=how)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held", [([1, 1], [5000, 3]), ([2, 1, 1], [2999, 4097, 1]), ([300], [1700])])
def test_attend_long(dtype, lens, held):
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 64)
    cache = make_cache(2, 64, 128, n_pages, table, seed=3)
    check_attend(cache, lens, held, table, randn(8, sum(lens), 8, 128).to(DT[dtype]), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held", [([1, 1, 1, 1], [200, 63, 10, 64]), ([80, 90, 3, 33], [120, 0, 7, 40])])
def test_attend_leaves_holes_out(dtype, lens, held):
    """Holes inside, at both ends and everywhere; the pages nobody holds have scales that are NaN."""
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 16)
    table[0, 1] = -1
    table[0, 5:7] = n_pages + 5
    table[1, 0] = -1
    table[2, :] = -1
    table[3, 2] = -3
    cache = make_cache(2, 16, 64, n_pages, table, seed=3)
    for s in (cache.k_scales, cache.v_scales):
        s[0] = float("nan")
        s[n_pages - 1] = float("nan")
    q = randn(8, sum(lens), 8, 64).to(DT[dtype])
    out = check_attend(cache, lens, held, table, q, dtype)
    assert bool((out[sum(lens[:2]):sum(lens[:3])] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1, 1], [40, 60]])
def test_attend_wide_ranges(dtype, lens):
    """Scores of hundreds, scales from 1e-30 to 1e4 side by side, a page of zeros (scale 0), queries of
    very different size, a negative softmax scale."""
    held = [300, 77]
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 16)
    cache = make_cache(2, 16, 64, n_pages, table, seed=3)
    cache.v_scales[table[0, 3]] = 1e4
    cache.v_scales[table[0, 5]] = 1e-30
    cache.v_scales[table[1, 0]] = 1e-30
    cache.v_scales[table[0, 0]] = 0.0
    cache.v_pages[table[0, 0]] = 0
    cache.k_scales[table[0, 2]] = 0.0
    cache.k_pages[table[0, 2]] = 0
    q = randn(8, sum(lens), 4, 64) * torch.logspace(-6, 1, sum(lens), device="cuda").view(-1, 1, 1)
    check_attend(cache, lens, held, table, q.to(DT[dtype]), dtype)
    check_attend(cache, lens, held, table, q.to(DT[dtype]), dtype, scale=-0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1, 1, 1], [50, 60, 40]])
def test_attend_keeps_nan_to_its_rows(dtype, lens):
    """A NaN query makes its own rows NaN; a NaN scale makes the rows that reach its page NaN."""
    held = [100, 64, 3]
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 16)
    cache = make_cache(2, 16, 64, n_pages, table, seed=3)
    q = randn(8, sum(lens), 4, 64).to(DT[dtype])
    batch, cu = batch_of(lens, held)
    clean, out = torch.empty_like(q), torch.empty_like(q)
    scd.scd_cache_attend(cache, batch, q, clean)
    q[0, 1, 5] = float("nan")
    cache.k_scales[table[1, 1], 0] = float("nan")
    cache.v_scales[table[1, 2], 1] = float("nan")
    scd.scd_cache_attend(cache, batch, q, out)
    bad = torch.isnan(out)
    want = torch.zeros_like(bad)
    want[0, 1] = True
    want[cu[1]:cu[2], :2] = True
    want[cu[1]:cu[2], 2:] = True
    assert torch.equal(bad, want)
    assert torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("n_seqs", [63, 64, 65, 300, 1000])
def test_many_requests(n_seqs):
    """More requests than a wave's or a workgroup's share of boundaries, many of them empty."""
    rng = np.random.default_rng(n_seqs)
    lens = rng.integers(0, 3, n_seqs).tolist()
    held = rng.integers(0, 40, n_seqs).tolist()
    table, n_pages = table_of(rng, lens, held, 16)
    cache = make_cache(1, 16, 32, n_pages, table, seed=3)
    batch, cu = batch_of(lens, held)
    t = sum(lens)
    k, v, q = randn(1, t, 1, 32), randn(2, t, 1, 32), randn(3, t, 2, 32)
    rot = scd.scd_rotary_table(scd.Rotary(32, 1e4), 64)
    before = state(cache)
    scd.scd_cache_append(cache, batch, k, v, rot)
    w = O.frequencies(32, 1e4)
    check_append(cache, before, table, cu, held, (O.rotate(f64(k), positions(lens, held), w), f64(v)))
    out = torch.empty_like(q)
    scd.scd_rotary(rot, batch, q, None, out, None)
    assert np.allclose(f64(out), O.rotate(f64(q), positions(lens, held), w), atol=1e-6)
    check_attend(cache, lens, held, table, q, "f32")


def test_pages_past_two_gigabytes():
    """Byte offsets that pass 32 bits: pages at both ends of pools of 2.3 GB."""
    n_pages = 140000
    table = np.array([[n_pages - 1, 0, n_pages - 2], [1, 131072, 131071]])
    pages = [torch.empty(n_pages, 1, 128, 128, dtype=torch.int8, device="cuda") for _ in "kv"]
    scales = [torch.zeros(n_pages, 1, device="cuda") for _ in "kv"]
    cache = scd.PagedCache(*pages, *scales, ints(table))
    lens, held = [300, 260], [0, 0]
    batch, cu = batch_of(lens, held)
    k, v = randn(1, 560, 1, 128).bfloat16(), randn(2, 560, 1, 128).bfloat16()
    scd.scd_cache_append(cache, batch, k, v)
    small = scd.PagedCache(*[torch.empty(6, 1, 128, 128, dtype=torch.int8, device="cuda") for _ in "kv"],
                           *[torch.zeros(6, 1, device="cuda") for _ in "kv"], ints([[0, 1, 2], [3, 4, 5]]))
    scd.scd_cache_append(small, batch, k, v)
    q = randn(3, 560, 4, 128).bfloat16()
    got, want = [torch.empty_like(q) for _ in range(2)], [torch.empty_like(k) for _ in range(4)]
    for c, o, kk, vv in ((cache, got[0], *want[:2]), (small, got[1], *want[2:])):
        scd.scd_cache_attend(c, batch, q, o)
        scd.scd_cache_read(c, batch, kk, vv)
    assert torch.equal(got[0], got[1]) and torch.equal(want[0], want[2]) and torch.equal(want[1], want[3])
    assert float((want[0].float() - k.float()).abs().max()) < 0.05


def test_same_bits_again_and_on_another_stream():
    lens, held = [1, 40, 1, 1], [3000, 20, 0, 700]
    table, n_pages = table_of(np.random.default_rng(4), lens, held, 64)
    cache = make_cache(2, 64, 128, n_pages, table, seed=3)
    batch, _ = batch_of(lens, held)
    q = randn(8, sum(lens), 8, 128).bfloat16()
    outs = [torch.empty_like(q) for _ in range(3)]
    call = scd.prepare_cache_attend(cache, batch, q, outs[0])
    call()
    first = outs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o in outs[1:]:
        scd.scd_cache_attend(cache, batch, q, o, stream=side)
    side.synchronize()
    for _ in range(3):
        call()
    assert torch.equal(first, outs[0]) and torch.equal(first, outs[1]) and torch.equal(first, outs[2])


def test_captured_steps_follow_growing_lengths():
    """One captured step (rotary, append, attend) replayed while the positions in device memory grow
    is what eager calls give."""
    n, heads, kv_heads, d, size = 3, 8, 2, 64, 16
    start = [5, 30, 100]
    table = ints(np.arange(1, 1 + n * 12).reshape(n, 12))
    rot = scd.scd_rotary_table(scd.Rotary(d, 1e4), 256)
    steps = [tuple(randn(100 * i + j, n, h, d).bfloat16() for j, h in enumerate((heads, kv_heads, kv_heads)))
             for i in range(20)]

    def world():
        gen = torch.Generator().manual_seed(9)
        pages = [torch.randint(-127, 128, (40, kv_heads, size, d), generator=gen, dtype=torch.int8).cuda() for _ in "kv"]
        scales = [torch.full((40, kv_heads), 0.02, device="cuda") for _ in "kv"]
        cache = scd.PagedCache(*pages, *scales, table)
        q, k, v = (torch.empty_like(x) for x in steps[0])
        pos0 = ints(start)
        batch = scd.Batch(n, ints(list(range(n + 1))), pos0)
        turned, out = torch.empty_like(q), torch.empty_like(q)
        calls = [scd.prepare_rotary(rot, batch, q, None, turned, None),
                 scd.prepare_cache_append(cache, batch, k, v, rot),
                 scd.prepare_cache_attend(cache, batch, turned, out)]
        return cache, (q, k, v), pos0, out, calls

    eager, graphed = world(), world()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for call in graphed[4]:
            call()
    for step in steps:
        for w in (eager, graphed):
            for dst, src in zip(w[1], step):
                dst.copy_(src)
        for call in eager[4]:
            call()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager[3], graphed[3])
        for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
            assert torch.equal(getattr(eager[0], name), getattr(graphed[0], name))
        eager[2].add_(1)
        graphed[2].add_(1)
