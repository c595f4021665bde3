"""Attention over latents and over dense rows, value by value within the roundings that it takes: nothing lost, nothing
counted twice, weights of 16 bits except where a call rounds them once."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from synth import workloads as W
from tests import attend_error as E
from tests import parity_util as U
from tests.latent_util import DT, f64, ints, randn
from tests.test_gpu_latent import SHAPES
from tests.test_gpu_latent import Case as Latent
from tests.test_gpu_rows import Case as Rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


def _latent_close(c, got=None):
    want, off = E.latent_attend(c.dtype, f64(c.pages), np.array(c.table), c.cu, c.held, f64(c.q), f64(c.w_k), f64(c.w_v),
                                c.scale)
    E.assert_close(f64(c.attend() if got is None else got), want, off)


def _rows_close(c, got=None):
    # calls of more than 64 query rows a KV head and request, of 16-byte rows, round weights once
    rows, wide = c.q.shape[0] * c.q.shape[1] // c.k.shape[1], all(s * x.element_size() % 16 == 0
                                                                  for x in (c.k, c.v) for s in x.stride()[:2])
    once = wide and -(-rows // min(c.batch.n_seqs, c.q.shape[0])) > 64
    want, off = E.rows_attend(c.dtype, c.cu, c.pos0, c.held_cu, c.first, f64(c.q), f64(c.k), f64(c.v), c.scale, once)
    E.assert_close(f64(c.attend() if got is None else got), want, off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("lens,held", [([1], [332]), ([1] * 5, [0, 63, 64, 127, 640]), ([37], [100])])
def test_latent(dtype, shape, lens, held):
    heads, plain, value, r, dr, page = shape
    _latent_close(Latent(dtype, lens, held, heads, plain, value, r, dr, page))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,held", [([1], [20000]), ([1] * 6, [9000, 1, 300, 5000, 64, 2500]), ([6, 1], [3000, 4000]),
                                       ([1] * 40, list(range(0, 2000, 50))), ([200], [500])])
def test_latent_cut(dtype, lens, held):
    """Tiles cut into many shares, some of one block."""
    _latent_close(Latent(dtype, lens, held, heads=6, plain=32, value=32, r=128, dr=32, page=16))


@pytest.mark.parametrize("dtype,r", [("bf16", 64), ("bf16", 256), ("bf16", 512), ("f32", 64), ("f32", 384)])
@pytest.mark.parametrize("rows", [1, 17, 33, 64, 65, 129, 300])
def test_latent_rows_of_a_tile(dtype, r, rows):
    _latent_close(Latent(dtype, [rows], [90], heads=1, plain=32, value=32, r=r, dr=32, page=32))
    _latent_close(Latent(dtype, [1, 1], [90, 20], heads=rows, plain=32, value=32, r=r, dr=32, page=32))


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_latent_scales(dtype, scale):
    c = Latent(dtype, [2, 1], [200, 31])
    c.scale = scale
    _latent_close(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,key,value", [
    (4, 4, 192, 128), (4, 2, 128, 128), (7, 1, 64, 64), (2, 2, 96, 64), (3, 3, 160, 96), (2, 1, 32, 32), (4, 4, 64, 128),
    (4, 1, 192, 64)])
@pytest.mark.parametrize("lens,pos0", [([1], [500]), ([130], [0]), ([5, 0, 1, 300], [62, 9, 1000, 0]),
                                       ([1] * 20, list(range(0, 400, 20)))])
def test_rows(dtype, heads, kv_heads, key, value, lens, pos0):
    _rows_close(Rows(dtype, lens, pos0, heads=heads, kv_heads=kv_heads, key=key, value=value))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 17, 64, 127, 700])
@pytest.mark.parametrize("group", [1, 3])
def test_rows_of_a_tile(dtype, tokens, group):
    _rows_close(Rows(dtype, [tokens], [77], heads=2 * group, kv_heads=2, key=64, value=64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_long(dtype):
    _rows_close(Rows(dtype, [1, 2, 1], [9000, 30, 4000], heads=8, kv_heads=2, key=128, value=128))


def test_rows_many_tiles():
    """None of them cut, the last ones first."""
    _rows_close(Rows("bf16", [900, 1100], [0, 50], heads=32, kv_heads=32, key=64, value=64))


# ---- long shares -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,least,most", [(512, 17000, 17800), (260, 39000, 40000)])
@pytest.mark.parametrize("poison", [False, True])
def test_latent_shares_of_many_pages(dtype, n, least, most, poison):
    """Shares of more than 1024 columns of the table, which are looked up a window at a time: a token of 512 requests
    (tiles that are not cut) and of 260 (cut in two), all naming the same pages; holes around the windows' ends."""
    heads, plain, value, r, dr, page = 2, 32, 32, 32, 32, 16
    tiles = n  # of 16 rows: a token of two heads each
    assert tiles >= 512 or -(-most // page) // 2 > 1024
    cols = -(-most // page)
    row = np.random.default_rng(n).permutation(np.arange(1, cols + 1))  # page 0 belongs to nobody
    for hole in (0, 3, 1015, 1016, 1019, 1021, 1023, 1024, 1025, 1028, 1032, cols // 2 + 1, cols // 2 + 1025, cols - 2):
        if hole < cols:
            row[hole] = -1
    held = np.random.default_rng(n + 1).integers(least, most - 1, n)
    held[0], held[-1] = most - 1, least
    pages = randn(1, cols + 1, page, r + dr).to(DT[dtype])
    pages[0] = float("nan") if poison else 0.0
    cache = scd.LatentCache(pages, ints(np.tile(row, (n, 1))), r)
    w_k, w_v = (randn(i, heads, 32, r).to(DT[dtype]) * r ** -0.5 for i in (2, 3))
    q = randn(4, n, heads, plain + dr).to(DT[dtype])
    out = torch.full((n, heads, value), float("nan"), dtype=DT[dtype], device="cuda")
    scale = 2.0 * (plain + dr) ** -0.5
    scd.scd_latent_attend(cache, scd.Batch(n, ints(np.arange(n + 1)), ints(held)), q, w_k, w_v, out, scale=scale)
    there = np.repeat(row >= 0, page)
    rows = np.where(there[:, None], f64(pages)[np.maximum(row, 0)].reshape(cols * page, -1), 0)
    seen = there[None] & (np.arange(cols * page)[None] <= held[:, None])
    some = np.concatenate([np.arange(0, n, 8), [n - 1]])  # the oracle's time
    want, off = E.over_latents(dtype, rows, seen[some], f64(q)[some], f64(w_k), f64(w_v), scale)
    E.assert_close(f64(out)[some], want, off)


# ---- what may hold anything --------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_latent_holes_beside_a_first_page_that_is_not_finite(dtype, bad):
    """Page 0 belongs to no request and holds anything; the first, a middle and the last visible column are holes."""
    c = Latent(dtype, [40, 1, 3], [30, 77, 150], heads=3, page=16)
    c.table = [[p + 1 if p >= 0 else -1 for p in row] for row in c.table]
    c.pages = torch.cat([torch.ones_like(c.pages[:1]), c.pages])
    for b, col in ((0, 2), (0, 4), (1, 0), (1, 4), (2, 5), (2, 9)):
        c.table[b][col] = -1
    c.caches()
    clean = c.attend()
    _latent_close(c, clean)
    c.pages[0] = bad
    assert torch.equal(c.attend(), clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_latent_not_finite_where_seen(dtype, bad):
    """Token 50 of a request that 40 rows attend to from position 30 on: it reaches rows 20 to 39, all of their values."""
    c = Latent(dtype, [40, 1], [30, 77], heads=3, page=16)
    clean = c.attend()
    c.pages[c.table[0][50 // 16], 50 % 16, 5] = bad
    got = c.attend()
    assert torch.equal(got[:20], clean[:20]) and torch.equal(got[40:], clean[40:])
    assert not torch.isfinite(got[20:40]).any()


# ---- dense rows as they lie --------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,pos0,group", [([3, 5], [400, 700], 2), ([100, 120], [380, 600], 2), ([1], [1200], 1)])
def test_rows_of_16_bytes_past_4_gib(dtype, lens, pos0, group):
    """Rows 2^21 elements apart, which are fetched 16 bytes at a time: the last ones lie behind 4 GiB."""
    c = Rows(dtype, lens, pos0, heads=2 * group, kv_heads=2, key=96, value=64)
    apart = 1 << 21
    assert (c.k.shape[0] - 1) * apart * c.k.element_size() > 1 << 32

    def far(x):
        t, h, d = x.shape
        y = torch.empty(t * apart, dtype=x.dtype, device="cuda").as_strided((t, h, d), (apart, d, 1))
        y.copy_(x)
        return y
    near = c.attend()
    _rows_close(c, near)
    assert torch.equal(c.attend(k=far(c.k), v=far(c.v)), near)


@pytest.mark.parametrize("name,layers", [("SMALL_BF16", (0, 1, 3, 4)), ("SMALL_F32", (0, 2))])
def test_rows_that_decode_and_patch_wrote(name, layers):
    """The codec's caches of Reuse and Patch layers, [tokens, heads * head_dim], read as they are."""
    wl = getattr(W, name)
    inp = U.Inputs(wl, "cuda")
    out = U.run_gpu(wl, inp, scd.scd_rope_table(U.model_of(wl), wl.max_position), which=("decode", "patch"))
    total = np.diff(wl.cu_seqlens).tolist()
    for new in ([1] * len(total), [min(n, 70 + 40 * b) for b, n in enumerate(total)]):
        c = Rows(wl.dtype, new, [a - b for a, b in zip(total, new)], heads=4 * wl.n_kv_heads, kv_heads=wl.n_kv_heads,
                 key=wl.head_dim, value=wl.head_dim)
        for layer in layers:
            c.k, c.v = (out[x][layer].view(-1, wl.n_kv_heads, wl.head_dim) for x in ("k_cache", "v_cache"))
            _rows_close(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_nobody(dtype):
    """Requests none of which holds a row."""
    c = Rows(dtype, [3, 90], [5, 0], rows=[0, 0], heads=4, kv_heads=2)
    assert c.k.shape[0] == 0 and not c.attend().any()
