"""The latent cache, attention over it and its expansion, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import latent_oracle as L
from oracle import serving_oracle as O
from tests.latent_util import DT, HALF, attend_bound, batch_of, f64, ints, paged, randn, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


class Case:
    """A cache, its requests, the heads' matrices and a query row for every new token."""

    def __init__(self, dtype, lens, held, heads=4, plain=64, value=64, r=64, dr=32, page=16, seed=0, spare=3, cols=None):
        self.dtype, self.lens, self.held, self.r, self.dr = dtype, lens, held, r, dr
        dt = DT[dtype]
        total = [n + h for n, h in zip(lens, held)]
        self.table, n_pages = paged(total, page, seed, spare, cols)
        self.pages = randn(seed + 1, n_pages, page, r + dr).to(dt)
        self.w_k = (randn(seed + 2, heads, plain, r) * r ** -0.5).to(dt)
        self.w_v = (randn(seed + 3, heads, value, r) * r ** -0.5).to(dt)
        self.batch, self.cu = batch_of(lens, held)
        self.q = randn(seed + 4, self.cu[-1], heads, plain + dr).to(dt)
        self.scale = 2.0 * (plain + dr) ** -0.5
        self.terms = plain + r + dr + max(total) + 64
        self.caches()

    def caches(self):
        self.cache = scd.LatentCache(self.pages, ints(self.table), self.r)

    def out(self):
        return torch.full((self.cu[-1], self.w_v.shape[0], self.w_v.shape[1]), float("nan"), dtype=DT[self.dtype],
                          device="cuda")

    def attend(self, out=None, q=None, **kw):
        out = self.out() if out is None else out
        scd.scd_latent_attend(self.cache, self.batch, self.q if q is None else q, self.w_k, self.w_v, out,
                              scale=self.scale, **kw)
        return out

    def want(self):
        return L.latent_attend(f64(self.pages), np.array(self.table), self.cu, self.held, f64(self.q), f64(self.w_k),
                               f64(self.w_v), self.scale)

    def check(self, got):
        want, mass, loud = self.want()
        off = np.abs(f64(got) - want)
        bound = attend_bound(self.dtype, want, mass, loud, self.terms)
        worst = np.unravel_index(np.argmax(off / bound), off.shape)
        assert np.all(off <= bound), (worst, off[worst], bound[worst])
        return want


# ---- append ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rotary_dim", [("half", 32), ("interleaved", 32), ("half", 16), ("interleaved", 10), (None, 0)])
@pytest.mark.parametrize("r,dr,page,how", [(64, 32, 16, "dense"), (96, 64, 32, "fused"), (256, 64, 128, "odd"),
                                           (512, 32, 64, "dense")])
def test_append(dtype, layout, rotary_dim, r, dr, page, how):
    lens, held = [3, 0, 1, 70, 1], [0, 5, 400, 17, 15]
    c = Case(dtype, lens, held, r=r, dr=dr, page=page)
    table = np.array(c.table)
    table[2, held[2] // page] = -1                  # a row without a page
    c.table = table.tolist()
    c.caches()
    t = c.cu[-1]
    rows = strided(randn(9, t + 2, 1, r + dr).to(DT[dtype]), how)[:t, 0]
    turns = None if layout is None else scd.scd_rotary_table(
        scd.Rotary(dr, 1e4, rotary_dim=rotary_dim, layout=layout, attention_factor=1.25), 500)
    want = f64(c.pages)
    w = None if layout is None else O.frequencies(rotary_dim, 1e4)
    L.append(want, table, c.cu, held, f64(rows[:, :r]), f64(rows[:, r:]), w, layout or "half", 1.25)
    scd.scd_latent_append(c.cache, c.batch, rows[:, :r], rows[:, r:], turns)
    got = f64(c.pages)
    assert np.array_equal(got[..., :r], want[..., :r])
    # two products and a sum of fp32 factors (4 roundings of at most 1.25 sqrt(2) times the pair), one to the type
    amp = 1.25 * 1.5 * np.abs(f64(rows)).max()
    assert np.all(np.abs(got - want) <= 1.01 * HALF[dtype] * np.abs(want) + 4 * 2.0 ** -24 * amp)


def test_append_leaves_rows_alone():
    """Behind the last request, past the table, in front of it: nothing is written."""
    c = Case("bf16", [4, 3], [14, 30], page=16, cols=2)
    before = c.pages.clone()
    batch = scd.Batch(9, ints([0, 4, 7]), ints([14, 30]))
    rows = randn(3, 9, c.r + c.dr).bfloat16()
    scd.scd_latent_append(c.cache, batch, rows[:, :c.r], rows[:, c.r:])
    want = f64(before)
    L.append(want, np.array(c.table), [0, 4, 7], [14, 30], f64(rows[:, :c.r]), f64(rows[:, c.r:]))
    assert np.array_equal(f64(c.pages), want)
    kept = c.pages.clone()
    scd.scd_latent_append(c.cache, scd.Batch(9, ints([0, 4, 7]), ints([-40, 32])), rows[:, :c.r], rows[:, c.r:])
    assert torch.equal(c.pages, kept)


# ---- attention ---------------------------------------------------------------------------------------------
SHAPES = [  # heads, plain, value, latent, turned, page
    (4, 64, 64, 64, 32, 16), (28, 128, 128, 96, 64, 64), (32, 128, 128, 256, 64, 64), (16, 64, 128, 512, 64, 32),
    (64, 128, 128, 128, 64, 128), (1, 32, 32, 32, 32, 16), (5, 96, 160, 160, 32, 32), (40, 256, 256, 384, 64, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("lens,held", [
    ([1], [0]), ([1], [332]), ([1, 1, 1], [0, 63, 64]), ([1] * 9, [0, 1, 15, 16, 31, 33, 200, 127, 640]),
    ([5, 0, 1, 3], [62, 9, 1000, 0]), ([37], [100]), ([0, 70, 2], [0, 0, 129])])
def test_attend(dtype, shape, lens, held):
    heads, plain, value, r, dr, page = shape
    c = Case(dtype, lens, held, heads, plain, value, r, dr, page)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held", [([1], [20000]), ([1] * 6, [9000, 1, 300, 5000, 64, 2500]), ([6, 1], [3000, 4000]),
                                       ([1] * 40, list(range(0, 2000, 50))), ([200], [500])])
def test_attend_long(dtype, lens, held):
    """Tiles cut into many shares, some of one block; windows of the page table that move on."""
    c = Case(dtype, lens, held, heads=6, plain=32, value=32, r=128, dr=32, page=16)
    c.check(c.attend())


@pytest.mark.parametrize("rows", [1, 3, 16, 17, 32, 33, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("dtype,r", [("bf16", 64), ("bf16", 256), ("bf16", 512), ("f32", 64)])
def test_attend_rows_of_a_tile(dtype, r, rows):
    """Every number of query rows a tile can hold, of one head and of many."""
    c = Case(dtype, [rows], [90], heads=1, plain=32, value=32, r=r, dr=32, page=32)
    c.check(c.attend())
    c = Case(dtype, [1, 1], [90, 20], heads=rows, plain=32, value=32, r=r, dr=32, page=32)
    c.check(c.attend())


@pytest.mark.parametrize("how", ["fused", "heads_first", "odd"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_strides(dtype, how):
    c = Case(dtype, [3, 1], [40, 99], heads=3)
    plain = c.attend()
    out = strided(c.out(), how)
    c.attend(out, q=strided(c.q, how))
    assert torch.equal(out, plain)


@pytest.mark.parametrize("scale", [0.0, -0.3, 25.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_scales(dtype, scale):
    c = Case(dtype, [2, 1], [200, 31])
    c.scale = scale
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_attend_masked_values(dtype, bad):
    """What no row may see holds values that are not finite: later tokens, holes, slots behind the last, other pages."""
    c = Case(dtype, [40, 1], [30, 77], heads=3, page=16)
    clean = c.attend()
    for b, n in enumerate((70, 78)):
        last = c.table[b][n // 16] if n // 16 < len(c.table[b]) else -1
        if last >= 0:
            c.pages[last, n % 16:] = bad
    used = {p for row in c.table for p in row}
    for p in range(c.pages.shape[0]):
        if p not in used:
            c.pages[p] = bad
    assert torch.equal(c.attend(), clean)
    # token 50 of the first request: rows before it do not see it, rows from it on do
    c.pages[c.table[0][50 // 16], 50 % 16, 5] = bad
    got = c.attend()
    assert torch.equal(got[:20], clean[:20]) and torch.equal(got[40:], clean[40:])
    if bad != bad:
        assert not torch.isfinite(got[20:40]).any()
    c.pages[c.table[0][50 // 16], 50 % 16, 5] = 0
    # a hole in the middle, whose page (0) holds anything
    c.table[1][2] = -1
    c.caches()
    c.pages[0 if 0 not in used else c.table[0][4], 0, 0] = c.pages[0, 0, 0]
    got = c.attend()
    want = L.latent_attend(np.nan_to_num(f64(c.pages), nan=0, posinf=0, neginf=0), np.array(c.table), c.cu, c.held,
                           f64(c.q), f64(c.w_k), f64(c.w_v), c.scale)
    bound = attend_bound(dtype, *want, c.terms)
    assert np.all((np.abs(f64(got) - want[0]) <= bound)[40:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_empty_rows(dtype):
    """Requests all of whose pages are holes, and positions in front of the first: zero rows."""
    c = Case(dtype, [2, 3, 1], [20, 40, 64])
    c.table[1] = [-1] * len(c.table[1])
    c.table[2][0], c.table[2][3] = 10 ** 6, -7
    c.caches()
    got = c.attend()
    c.check(got)
    assert not got[2:5].any()
    got = c.out()
    scd.scd_latent_attend(c.cache, scd.Batch(6, ints([0, 2, 5, 6]), ints([-1, -9, 3])), c.q, c.w_k, c.w_v, got)
    assert not got[0].any() and got[1].any() and not got[2:5].any()


def test_attend_rows_behind_the_last_request():
    c = Case("bf16", [2, 1], [20, 40])
    q = randn(1, 6, 4, 96).bfloat16()
    q[:3] = c.q
    out = torch.full((6, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    scd.scd_latent_attend(c.cache, scd.Batch(6, ints([0, 2, 3]), ints([20, 40])), q, c.w_k, c.w_v, out, scale=c.scale)
    # one more row a request on average: another tile, the same rows of it
    c.check(out[:3])
    assert (out[3:] == 7).all()


def test_attend_past_the_table():
    """Positions that the table has no columns for are left out."""
    c = Case("bf16", [1, 4], [47, 29], cols=3)
    c.held = [100, 29]
    c.batch = scd.Batch(5, ints([0, 1, 5]), ints(c.held))
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_graph(dtype):
    """Captured once, replayed while lengths grow; two graphs share a workspace one after another."""
    c = Case(dtype, [1, 1, 1], [700, 33, 2], heads=8)
    pos0 = ints(c.held)
    batch = scd.Batch(3, ints([0, 1, 2, 3]), pos0)
    ws = torch.full((scd.scd_latent_attend_workspace_bytes(c.cache, batch, 8),), 255, dtype=torch.uint8, device="cuda")
    outs = [c.out(), c.out()]
    calls = [scd.prepare_latent_attend(c.cache, batch, q, c.w_k, c.w_v, o, scale=c.scale, workspace=ws)
             for q, o in ((c.q, outs[0]), (-c.q, outs[1]))]
    for call in calls:
        call()
    graphs = []
    for call in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for held in ([0, 0, 0], [1, 17, 0], [650, 32, 2], [700, 33, 1]):
        pos0.copy_(ints(held))
        c.held = held
        for o in outs:
            o.fill_(float("nan"))
        for g in graphs:
            g.replay()
        c.check(outs[0])
        eager = scd.prepare_latent_attend(c.cache, batch, -c.q, c.w_k, c.w_v, c.out(), scale=c.scale)
        eager()
        assert torch.equal(eager._keep[-2], outs[1])
        torch.cuda.synchronize()


def test_attend_on_another_stream():
    c = Case("bf16", [1] * 4, [900, 3, 64, 250], heads=16)
    want = c.attend()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = c.out()
    s.wait_stream(torch.cuda.current_stream())
    c.attend(out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


def test_attend_repeats():
    c = Case("bf16", [3] * 7, [2000, 1, 64, 333, 900, 17, 128], heads=12, r=96)
    first = c.attend()
    for _ in range(5):
        assert torch.equal(c.attend(), first)


# ---- expansion ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("lens,pos0", [([1], [0]), ([130, 0, 3], [0, 4, 50]), ([63, 65], [1, 0])])
@pytest.mark.parametrize("how", ["dense", "odd"])
def test_expand(dtype, shape, lens, pos0, how):
    heads, plain, value, r, dr, page = shape
    c = Case(dtype, lens, pos0, heads, plain, value, r, dr, page)
    if len(lens) == 3:
        c.table[0][1 % len(c.table[0])] = -1
        c.caches()
    t = c.cu[-1] + 2
    batch = scd.Batch(t, ints(c.cu), ints(pos0))
    k, v = (strided(torch.full((t, heads, d), 7.0, dtype=DT[dtype], device="cuda"), how) for d in (plain + dr, value))
    scd.scd_latent_expand(c.cache, batch, c.w_k, c.w_v, k, v)
    assert (k[-2:] == 7).all() and (v[-2:] == 7).all()
    want = L.expand(f64(c.pages), np.array(c.table), c.cu, pos0, f64(c.w_k), f64(c.w_v))
    loud = L.expand(np.abs(f64(c.pages)), np.array(c.table), c.cu, pos0, np.abs(f64(c.w_k)), np.abs(f64(c.w_v)))
    for x, y, a in zip((k, v), want, loud):
        assert np.all(np.abs(f64(x[:-2]) - y) <= 1.01 * HALF[dtype] * np.abs(y) + r * 2.0 ** -24 * a)
    assert np.array_equal(f64(k[:-2, :, plain:]), want[0][..., plain:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [32, 64, 96, 160, 256, 384])
def test_expand_keeps_rows_and_channels_apart(dtype, r):
    """A key or a latent that is not finite reaches its own row only, and a key no product."""
    c = Case(dtype, [70], [0], 2, 64, 32, r, 32, 16)
    k, v = (torch.empty(70, 2, d, dtype=DT[dtype], device="cuda") for d in (96, 32))
    scd.scd_latent_expand(c.cache, c.batch, c.w_k, c.w_v, k, v)
    clean = k.clone(), v.clone()
    c.pages[c.table[0][1], 3, r + 5] = float("nan")
    c.pages[c.table[0][2], 4, 7] = float("inf")
    scd.scd_latent_expand(c.cache, c.batch, c.w_k, c.w_v, k, v)
    assert torch.isnan(k[19, :, 69]).all()
    k[19, :, 69] = clean[0][19, :, 69]
    assert not torch.isfinite(k[36, :, :64]).any() and not torch.isfinite(v[36]).any()
    k[36], v[36] = clean[0][36], clean[1][36]
    assert torch.equal(k, clean[0]) and torch.equal(v, clean[1])


# ---- together ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_tokens(dtype):
    """A prompt appended, attended in both forms, and a token behind it."""
    heads, plain, value, r, dr, page = 4, 64, 64, 96, 32, 32
    lens = [150, 41]
    c = Case(dtype, lens, [0, 0], heads, plain, value, r, dr, page)
    turns = scd.scd_rotary_table(scd.Rotary(dr, 1e4), 200)
    rows = randn(5, c.cu[-1], r + dr).to(DT[dtype])
    scd.scd_latent_append(c.cache, c.batch, rows[:, :r], rows[:, r:], turns)
    tail = c.q[..., plain:]
    scd.scd_rotary(turns, c.batch, tail, None, tail, None)
    absorbed = c.attend()
    c.check(absorbed)
    k, v = (torch.empty(c.cu[-1], heads, d, dtype=DT[dtype], device="cuda") for d in (plain + dr, value))
    scd.scd_latent_expand(c.cache, c.batch, c.w_k, c.w_v, k, v)
    out = c.out()
    scd.scd_rows_attend(c.batch, c.batch, c.q, k, v, out, scale=c.scale)
    want, mass, loud = L.rows_attend(c.cu, [0, 0], c.cu, [0, 0], f64(c.q), f64(k), f64(v), c.scale)
    assert np.all(np.abs(f64(out) - want) <= attend_bound(dtype, want, mass, loud, c.terms))
    # the two forms differ by the rounding of the dense keys and values: a score's magnitudes times half a step
    want, mass, loud = c.want()
    slack = mass * (2 * (np.exp(HALF[dtype] * loud) - 1) + HALF[dtype])
    assert np.all(np.abs(f64(out) - want) <= attend_bound(dtype, want, mass, loud, c.terms) + slack)
