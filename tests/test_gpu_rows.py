"""Causal attention over dense rows, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import latent_oracle as L
from tests.latent_util import DT, attend_bound, batch_of, f64, ints, randn, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


class Case:
    def __init__(self, dtype, lens, pos0, rows=None, first=None, heads=4, kv_heads=2, key=64, value=64, seed=0):
        self.dtype, self.pos0 = dtype, pos0
        self.first = first or [0] * len(lens)
        rows = rows or [n + p - f for n, p, f in zip(lens, pos0, self.first)]
        self.batch, self.cu = batch_of(lens, pos0)
        self.held, self.held_cu = batch_of(rows, first)
        dt = DT[dtype]
        self.q = randn(seed, self.cu[-1], heads, key).to(dt)
        self.k, self.v = (randn(seed + 1, self.held_cu[-1], kv_heads, d).to(dt) for d in (key, value))
        self.scale = 2 * key ** -0.5
        self.terms = key + max(rows) + 64

    def out(self):
        return torch.full((self.cu[-1], self.q.shape[1], self.v.shape[2]), float("nan"), dtype=DT[self.dtype], device="cuda")

    def attend(self, out=None, q=None, k=None, v=None, **kw):
        out = self.out() if out is None else out
        scd.scd_rows_attend(self.batch, self.held, self.q if q is None else q, self.k if k is None else k,
                            self.v if v is None else v, out, scale=self.scale, **kw)
        return out

    def check(self, got):
        want, mass, loud = L.rows_attend(self.cu, self.pos0, self.held_cu, self.first, f64(self.q), f64(self.k),
                                         f64(self.v), self.scale)
        off, bound = np.abs(f64(got) - want), attend_bound(self.dtype, want, mass, loud, self.terms)
        worst = np.unravel_index(np.argmax(off / bound), off.shape)
        assert np.all(off <= bound), (worst, off[worst], bound[worst])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,key,value", [
    (4, 4, 192, 128), (4, 2, 128, 128), (7, 1, 64, 64), (2, 2, 96, 64), (3, 3, 160, 96), (2, 1, 32, 32), (4, 4, 64, 128),
    (4, 1, 192, 64)])
@pytest.mark.parametrize("lens,pos0", [([1], [0]), ([1], [500]), ([130], [0]), ([5, 0, 1, 300], [62, 9, 1000, 0]),
                                       ([64, 65, 1], [0, 64, 63]), ([1] * 20, list(range(0, 400, 20)))])
def test_attend(dtype, heads, kv_heads, key, value, lens, pos0):
    c = Case(dtype, lens, pos0, heads=heads, kv_heads=kv_heads, key=key, value=value)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 2, 16, 17, 31, 64, 127, 128, 129, 700])
@pytest.mark.parametrize("group", [1, 3])
def test_attend_rows_of_a_tile(dtype, tokens, group):
    c = Case(dtype, [tokens], [77], heads=2 * group, kv_heads=2, key=64, value=64)
    c.check(c.attend())


def test_attend_many_tiles():
    """So many tiles that none is cut, the last ones first."""
    c = Case("bf16", [900, 1100], [0, 50], heads=32, kv_heads=32, key=64, value=64)
    assert scd.scd_rows_attend_workspace_bytes(c.batch, c.held, torch.bfloat16, 32, 32, 64, 64) == 0
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_long(dtype):
    c = Case(dtype, [1, 2, 1], [9000, 30, 4000], heads=8, kv_heads=2, key=128, value=128)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_windows_and_empty_rows(dtype):
    """Rows that begin behind position 0 (a window), queries in front of all of them, requests without rows."""
    c = Case(dtype, [4, 3, 2, 5], [10, 0, 7, 100], rows=[12, 5, 0, 20], first=[2, 2, 0, 90], heads=2)
    got = c.attend()
    c.check(got)
    assert not got[4:6].any() and got[6].any() and not got[7:9].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["fused", "heads_first", "odd"])
def test_attend_strides(dtype, how):
    c = Case(dtype, [70, 3], [5, 90], heads=4, kv_heads=2, key=96, value=64)
    want = c.attend()
    c.check(want)
    for which in ("q", "k", "v", "all"):
        args = {n: strided(getattr(c, n), how) for n in "qkv" if which in (n, "all")}
        out = strided(c.out(), how if which == "all" else "dense")
        c.attend(out, **args)
        c.check(out)
        if which == "q" or how != "odd":  # other keys' and values' rows are read the same way
            assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_attend_masked_values(dtype, bad):
    c = Case(dtype, [100], [30], heads=4, kv_heads=2, key=64, value=64)
    clean = c.attend()
    for name in "kv":
        x = getattr(c, name).clone()
        x[80:, :, 3] = bad        # token 50 of the new ones on
        got = c.attend(**{name: x})
        assert torch.equal(got[:50], clean[:50])
        if name == "v":
            assert torch.isnan(got[50:, :, 3]).all()
            rest = [i for i in range(64) if i != 3]
            assert torch.equal(got[50:][..., rest], clean[50:][..., rest])
        elif bad != bad:
            assert torch.isnan(got[50:]).all()
    # rows of another request, and behind the last one
    k, v = (torch.cat([x, torch.full_like(x[:70], bad)]) for x in (c.k, c.v))
    out = c.out()
    scd.scd_rows_attend(c.batch, scd.Batch(200, ints([0, 130])), c.q, k, v, out, scale=c.scale)
    assert torch.equal(out, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_large_scores(dtype):
    c = Case(dtype, [40], [100])
    c.scale = 30.0
    c.check(c.attend())


def test_attend_rows_behind_the_last_request():
    c = Case("bf16", [3, 2], [40, 10])
    q = torch.cat([c.q, c.q])
    out = torch.full((10, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    scd.scd_rows_attend(scd.Batch(10, ints(c.cu), ints(c.pos0)), c.held, q, c.k, c.v, out, scale=c.scale)
    c.check(out[:5])
    assert (out[5:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_graph_and_stream(dtype):
    c = Case(dtype, [2, 30], [600, 0], heads=4, kv_heads=1)
    want = c.attend()
    out = c.out()
    call = scd.prepare_rows_attend(c.batch, c.held, c.q, c.k, c.v, out, scale=c.scale)
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    s = torch.cuda.Stream()
    out.fill_(float("nan"))
    s.wait_stream(torch.cuda.current_stream())
    c.attend(out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


def test_attend_the_codecs_caches():
    """The caches that decode and Patch write, [tokens, heads * head_dim], read as they are."""
    c = Case("bf16", [6], [120], heads=8, kv_heads=4, key=64, value=64)
    want = c.attend()
    k, v = c.k.reshape(126, 256), c.v.reshape(126, 256)
    assert torch.equal(c.attend(k=k.view(126, 4, 64), v=v.view(126, 4, 64)), want)
