"""The latent cache, dense rows and pages at the ends of their ranges and as programs run them: many requests, tensors
past 4 GiB, broadcast inputs, calls side by side, whole steps captured."""
import random

import numpy as np
import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import latent_oracle as L
from tests.latent_util import DT, HALF, attend_bound, f64, ints, randn
from tests.test_gpu_latent import Case as Latent
from tests.test_gpu_pages import Both
from tests.test_gpu_rows import Case as Rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


def _many(n, seed):
    """Requests of none, one and some tokens, the first and the last without any."""
    rng = random.Random(seed)
    lens = [0] + [rng.choice([0, 1, 1, 1, 2, 5]) for _ in range(n - 2)] + [0]
    return lens, [rng.choice([0, 1, 15, 16, 40, 90]) for _ in range(n)]


# ---- many requests -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [64, 65, 256, 257, 1100])
def test_latent_attend_many_requests(dtype, n):
    lens, held = _many(n, n)
    c = Latent(dtype, lens, held, heads=2, plain=32, value=32, r=32)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_latent_attend_many_requests_cut(dtype):
    """More requests than are planned at once, of which few have tokens: their positions are cut."""
    n = 600
    lens, held = [0] * n, [0] * n
    for b, t, h in ((3, 1, 900), (255, 2, 64), (256, 1, 1500), (400, 3, 0), (598, 1, 333)):
        lens[b], held[b] = t, h
    c = Latent(dtype, lens, held, heads=2, plain=32, value=32, r=32)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [65, 257, 1100])
def test_latent_append_and_expand_many_requests(dtype, n):
    lens, held = _many(n, n + 1)
    c = Latent(dtype, lens, held, heads=2, plain=32, value=32, r=32)
    rows = randn(9, c.cu[-1], c.r + c.dr).to(DT[dtype])
    want = f64(c.pages)
    L.append(want, np.array(c.table), c.cu, held, f64(rows[:, :c.r]), f64(rows[:, c.r:]))
    scd.scd_latent_append(c.cache, c.batch, rows[:, :c.r], rows[:, c.r:])
    assert np.array_equal(f64(c.pages), want)
    k, v = (torch.empty(c.cu[-1], 2, d, dtype=DT[dtype], device="cuda") for d in (32 + c.dr, 32))
    scd.scd_latent_expand(c.cache, c.batch, c.w_k, c.w_v, k, v)
    args = np.array(c.table), c.cu, held
    want = L.expand(f64(c.pages), *args, f64(c.w_k), f64(c.w_v))
    loud = L.expand(np.abs(f64(c.pages)), *args, np.abs(f64(c.w_k)), np.abs(f64(c.w_v)))
    for x, y, a in zip((k, v), want, loud):
        assert np.all(np.abs(f64(x) - y) <= 1.01 * HALF[dtype] * np.abs(y) + c.r * 2.0 ** -24 * a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [65, 257, 1100])
def test_rows_attend_many_requests(dtype, n):
    lens, held = _many(n, n + 2)
    c = Rows(dtype, lens, held, heads=2, kv_heads=1, key=32, value=32)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 40, 300])
def test_rows_attend_joins(dtype, tokens):
    """Positions that are cut, joined by four waves a row (to 1024 rows) and by one."""
    c = Rows(dtype, [tokens], [2000], heads=8, kv_heads=2, key=64, value=96)
    assert scd.scd_rows_attend_workspace_bytes(c.batch, c.held, DT[dtype], 8, 2, 64, 96) > 0
    c.check(c.attend())


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2500])
def test_reserve_many_requests(n):
    """Steps of a token as one workgroup's threads hold them, and of more requests than that."""
    rng = random.Random(n)
    b = Both(2 * n + 7, n, 4)
    b.reserve([rng.choice([1, 10, 16, 20]) for _ in range(n)])
    gone = rng.sample(range(n), n // 3)
    b.free(gone)
    left = [i for i in range(n) if b.pool.held[i]]
    b.fork([rng.choice(left) for _ in gone], gone)
    b.reserve([1] * n)
    b.compact()


def test_reserve_long_prompts_of_many_requests():
    """Columns of more requests than threads, shared pages among them; then calls that change nothing."""
    rng = random.Random(8)
    n = 1300
    b = Both(9000, n, 12)
    b.reserve([rng.choice([0, 1, 16, 17, 100, 150]) if i % 3 else 0 for i in range(n)])
    empty, full = ([i for i in range(n) if (b.pool.held[i] > 0) == held] for held in (False, True))
    b.fork([rng.choice(full) for _ in empty], empty)
    b.reserve([rng.choice([0, 1, 1, 5, 40]) for _ in range(n)])
    late = [0] * n
    late[1200] = 13 * 16
    assert b.reserve(late)[3] == 1
    assert b.reserve([12 * 16 - h for h in b.pool.held])[2] > 0
    b.free(rng.sample(range(n), 700))
    b.reserve([rng.choice([0, 1, 33]) if h < 150 else 0 for h in b.pool.held])
    b.compact()


# ---- past 4 GiB --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_latent_cache_past_4_gib(dtype):
    """The same requests in the first pages of a small pool and in the last ones of a large."""
    size, r, dr = 128, 512, 64
    c = Latent(dtype, [1, 3], [300, 129], heads=4, plain=32, value=32, r=r, dr=dr, page=size, spare=0)
    n, eb = c.pages.shape[0], c.pages.element_size()
    n_pages = (5 << 30) // (size * (r + dr) * eb) + n
    pages = torch.empty(n_pages, size, r + dr, dtype=DT[dtype], device="cuda")
    pages[-n:] = c.pages
    far = scd.LatentCache(pages, ints([[p + n_pages - n if p >= 0 else -1 for p in row] for row in c.table]), r)
    rows = randn(3, 4, r + dr).to(DT[dtype])
    for cache in (c.cache, far):
        scd.scd_latent_append(cache, c.batch, rows[:, :r], rows[:, r:])
    assert torch.equal(pages[-n:], c.pages)
    out = c.out()
    scd.scd_latent_attend(far, c.batch, c.q, c.w_k, c.w_v, out, scale=c.scale)
    assert torch.equal(out, c.attend())
    c.check(out)
    got = [[torch.empty(4, 4, d, dtype=DT[dtype], device="cuda") for d in (32 + dr, 32)] for _ in "ab"]
    for cache, (k, v) in zip((c.cache, far), got):
        scd.scd_latent_expand(cache, c.batch, c.w_k, c.w_v, k, v)
    for a, b in zip(*got):
        assert torch.equal(a, b)
    moves = scd.Moves(ints([[n_pages - 1, 1], [0, n_pages - 2]]), ints([2, 0, 0, 0]))
    pages[0] = 3
    last = pages[-1].clone()
    scd.scd_pages_copy([far], moves)
    assert torch.equal(pages[1], last) and (pages[-2] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [0, 1])
def test_dense_rows_past_4_gib(dtype, odd):
    """Rows far apart: the last ones, of the second request, begin behind 4 GiB."""
    c = Rows(dtype, [3, 5], [40, 100], heads=4, kv_heads=2, key=64, value=64)
    want = c.attend()
    eb = c.k.element_size()
    apart = (5 << 30) // (c.k.shape[0] * eb) // 8 * 8 + odd

    def far(x):
        t, h, d = x.shape
        y = torch.empty(t * apart, dtype=x.dtype, device="cuda").as_strided((t, h, d), (apart, d, 1))
        y.copy_(x)
        return y
    k, v = far(c.k), far(c.v)
    assert (c.k.shape[0] - 5) * apart * eb > 1 << 32
    got = c.attend(k=k, v=v)
    c.check(got)
    if not odd:
        assert torch.equal(got, want)


# ---- broadcast inputs --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_broadcast_inputs(dtype):
    """Rows and heads that share memory are read as if each had its own."""
    c = Latent(dtype, [2, 3], [70, 0], heads=4)
    one = c.q[:1].clone()
    assert torch.equal(c.attend(q=one.expand(5, -1, -1)), c.attend(q=one.repeat(5, 1, 1)))
    head = c.q[:, :1].clone()
    assert torch.equal(c.attend(q=head.expand(-1, 4, -1)), c.attend(q=head.repeat(1, 4, 1)))
    row = randn(5, 1, c.r + c.dr).to(DT[dtype]).expand(5, -1)
    scd.scd_latent_append(c.cache, c.batch, row[:, :c.r], row[:, c.r:])
    first = c.pages.clone()
    c.pages.zero_()
    whole = row.contiguous()
    scd.scd_latent_append(c.cache, c.batch, whole[:, :c.r], whole[:, c.r:])
    there = c.pages != 0
    assert there.any() and torch.equal(first[there], c.pages[there])
    d = Rows(dtype, [2, 3], [70, 0], heads=4, kv_heads=4)
    k, v = d.k[:, :1], d.v[:1]
    assert torch.equal(d.attend(k=k.expand(-1, 4, -1), v=v.expand(d.v.shape[0], -1, -1)),
                       d.attend(k=k.repeat(1, 4, 1), v=v.repeat(d.v.shape[0], 1, 1)))


# ---- side by side, captured ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_side_by_side(dtype):
    """Calls on two streams, each with a workspace of its own, as one after another."""
    a = Latent(dtype, [1] * 5, [900, 3, 64, 250, 1200], heads=16, seed=1)
    b = Latent(dtype, [4, 9], [1000, 31], heads=8, r=96, seed=2)
    d = Rows(dtype, [7, 40], [800, 100], heads=8, kv_heads=2, seed=3)
    want = [a.attend(), b.attend(), d.attend()]
    streams = [torch.cuda.Stream() for _ in want]
    outs = [x.out() for x in (a, b, d)]
    for _ in range(6):
        for o in outs:
            o.fill_(float("nan"))
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for x, o, s in zip((a, b, d), outs, streams):
            x.attend(o, stream=s)
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_step(dtype):
    """A step captured once: pages reserved and copied, a token appended, attended in both forms.  Lengths grow
    in device memory between replays; every replay against the same calls made eagerly on another pool."""
    size, heads, plain, value, r, dr, n, cols = 16, 4, 32, 32, 64, 32, 3, 4
    w_k, w_v = (randn(i, heads, 32, r).to(DT[dtype]) / 8 for i in (1, 2))
    turns = scd.scd_rotary_table(scd.Rotary(dr, 1e4), 64)
    cu, rows_cu = ints([0, 1, 2, 3]), ints([0] * 4)
    batch_rows = n * cols * size

    class Side:
        def __init__(self):
            self.table, self.held = ints([[-1] * cols] * n), ints([0] * n)
            self.pages = scd.Pages(self.table, ints([0] * 12), self.held, size)
            self.moves = scd.Moves(ints([[0, 0]] * 6), ints([0] * 4))
            data = torch.zeros(12, size, r + dr, dtype=DT[dtype], device="cuda")
            self.cache = scd.LatentCache(data, self.table, r)
            self.rows, self.q = torch.zeros(n, r + dr, dtype=DT[dtype], device="cuda"), \
                torch.zeros(n, heads, plain + dr, dtype=DT[dtype], device="cuda")
            self.k, self.v = (torch.zeros(batch_rows, heads, d, dtype=DT[dtype], device="cuda") for d in (plain + dr, value))
            self.a, self.o = (torch.zeros(n, heads, value, dtype=DT[dtype], device="cuda") for _ in "ao")
            self.new = scd.Batch(n, cu, self.held)
            self.whole = scd.Batch(batch_rows, rows_cu)
            tail = self.q[..., plain:]
            self.calls = [scd.prepare_pages_reserve(self.pages, self.new, self.moves),
                          scd.prepare_pages_copy([self.cache], self.moves),
                          scd.prepare_latent_append(self.cache, self.new, self.rows[:, :r], self.rows[:, r:], turns),
                          scd.prepare_rotary(turns, self.new, tail, None, tail, None),
                          scd.prepare_latent_attend(self.cache, self.new, self.q, w_k, w_v, self.a),
                          scd.prepare_latent_expand(self.cache, self.whole, w_k, w_v, self.k, self.v),
                          scd.prepare_rows_attend(self.new, self.whole, self.q, self.k, self.v, self.o)]

        def load(self, seed, held):
            self.held.copy_(ints(held))
            self.rows.copy_(randn(seed, n, r + dr))
            self.q.copy_(randn(seed + 1, n, heads, plain + dr))

    x, e = Side(), Side()
    graph = None
    for step in range(34):
        held = [step, step, step // 2]
        if step % 2:  # the third request takes its tokens every other step
            held[2] += 1
        rows_cu.copy_(ints(np.concatenate([[0], np.cumsum([h + 1 for h in held])])))
        for s in (x, e):
            s.load(10 * step, held)
        if graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                for call in x.calls:
                    call()
        graph.replay()
        for call in e.calls:
            call()
        torch.cuda.synchronize()
        for p, q in ((x.table, e.table), (x.pages.refs, e.pages.refs), (x.cache.pages, e.cache.pages), (x.a, e.a),
                     (x.o, e.o)):
            assert torch.equal(p, q), step
        if step in (0, 15, 16, 33):
            want, mass, loud = L.latent_attend(f64(x.cache.pages), x.table.cpu().numpy(), [0, 1, 2, 3], held, f64(x.q),
                                               f64(w_k), f64(w_v), (plain + dr) ** -0.5)
            bound = attend_bound(dtype, want, mass, loud, plain + r + dr + 64 + 64)
            assert np.all(np.abs(f64(x.a) - want) <= bound)
            slack = mass * (2 * (np.exp(HALF[dtype] * loud) - 1) + HALF[dtype])  # dense keys and values are rounded
            assert np.all(np.abs(f64(x.o) - want) <= bound + slack)
