"""Pages given back, shared, reserved, moved to the front and copied, against lists."""
import random

import pytest
import torch

import paper_2606_07684_amd as scd
from oracle import latent_oracle as L
from tests.latent_util import ints, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


class Both:
    """A pool on the device and as lists, with one small cache of each kind whose pages hold their own numbers."""

    def __init__(self, n_pages, n_seqs, cols, size=16):
        self.pool = L.Pool([[-1] * cols for _ in range(n_seqs)], [0] * n_pages, [0] * n_seqs, size)
        self.pages = scd.Pages(ints(self.pool.table), ints(self.pool.refs), ints(self.pool.held), size)
        self.moves = scd.Moves(torch.full((max(n_seqs, n_pages // 2), 2), -5, dtype=torch.int32, device="cuda"),
                               torch.full((4,), -5, dtype=torch.int32, device="cuda"))
        ids = torch.arange(n_pages, device="cuda")
        rows = ids.view(-1, 1, 1).expand(-1, size, 96).bfloat16().contiguous()
        kv = [(ids.view(-1, 1, 1, 1) % 100).expand(-1, 3, size, 32).to(torch.int8).contiguous() for _ in range(2)]
        scales = [ids.view(-1, 1).expand(-1, 3).float().contiguous() * f for f in (1.0, 2.0)]
        self.caches = [scd.LatentCache(rows, self.pages.page_table, 64), scd.PagedCache(*kv, *scales, self.pages.page_table)]
        self.planes = [rows, *kv, *scales]

    def load(self, table, held):
        self.pool.table = [list(r) for r in table]
        self.pool.held = list(held)
        self.pool.refs = [sum(p == q for r in table for q in r) for p in range(len(self.pool.refs))]
        for t, v in ((self.pages.page_table, self.pool.table), (self.pages.held, held), (self.pages.refs, self.pool.refs)):
            t.copy_(ints(v))

    def same(self):
        assert self.pages.page_table.tolist() == self.pool.table
        assert self.pages.refs.tolist() == self.pool.refs
        assert self.pages.held.tolist() == self.pool.held

    def free(self, seqs):
        scd.scd_pages_free(self.pages, ints(seqs))
        self.pool.free(seqs)
        self.same()

    def fork(self, src, dst):
        scd.scd_pages_fork(self.pages, ints(src), ints(dst))
        self.pool.fork(src, dst)
        self.same()

    def _moved(self, moves, status):
        assert self.moves.status.tolist() == status
        pairs = self.moves.pairs.tolist()
        assert [tuple(x) for x in pairs[:len(moves)]] == moves
        before = [t.clone() for t in self.planes]
        scd.scd_pages_copy(self.caches, self.moves)
        for was, now in zip(before, self.planes):
            for a, b in moves:
                was[b] = was[a]
            assert torch.equal(was, now)

    def reserve(self, new, advance=True):
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        scd.scd_pages_reserve(self.pages, scd.Batch(cu[-1], ints(cu)), self.moves)
        moves, status = self.pool.reserve(new)
        self.same()
        self._moved(moves, status)
        if advance and not status[2] and not status[3]:
            self.pool.held = [h + n for h, n in zip(self.pool.held, new)]
            self.pages.held.copy_(ints(self.pool.held))
        return status

    def compact(self):
        scd.scd_pages_compact(self.pages, self.moves)
        moves, status = self.pool.compact()
        self.same()
        self._moved(moves, status)


def test_life_of_a_search():
    b = Both(60, 6, 8)
    b.reserve([37, 0, 0, 100, 0, 0])
    b.fork([0, 0, 3], [1, 2, 4])
    assert b.reserve([1, 1, 1, 1, 1, 0])[0] == 3        # pages begun and shared: all but the last writer's
    b.reserve([1, 1, 1, 1, 1, 0])
    b.free([0, 4])
    b.fork([2, 3], [0, 5])
    assert b.reserve([20, 0, 0, 0, 0, 5])[0] == 2       # the sources do not write: both are copied
    b.free([1, 3, 2])
    b.compact()
    b.reserve([3, 30, 0, 0, 0, 1])
    b.free([0, 1, 2, 3, 4, 5])
    b.compact()
    assert b.pool.refs == [0] * 60


def test_forks_of_whole_pages_copy_nothing():
    b = Both(20, 4, 6)
    b.reserve([32, 0, 0, 0])
    b.fork([0, 0, 0], [1, 2, 3])
    assert b.reserve([1, 1, 1, 1])[0] == 0
    assert b.pool.table[0][:2] == b.pool.table[3][:2]


def test_fork_passes_over():
    b = Both(40, 8, 6)
    b.reserve([20, 17, 0, 0, 5, 0, 0, 0])
    # twice the same target, a target that holds pages, a source that is a target, out of range, itself, a target
    # that an earlier pair named in vain
    b.fork([0, 1, 0, 0, 2, 0, 9, -1, 3, 4], [2, 2, 1, 3, 5, 8, 6, 7, 3, 6])
    assert b.pool.held == [20, 17, 20, 20, 5, 0, 0, 0]
    b.fork([0, 5], [2, 7])
    assert b.pool.held[2] == 20 and b.pool.held[7] == 0


def test_free_passes_over():
    b = Both(40, 6, 6)
    b.reserve([40, 17, 33, 0, 5, 1])
    b.fork([0], [3])
    b.free([0, 0, -1, 6, 4, 0, 4])
    assert sum(b.pool.refs) == 3 + 2 + 3 + 1
    b.free([3, 3])
    b.pages.refs.zero_()  # counts that are too low stay at zero
    b.pool.refs = [0] * 40
    b.free([1])


def test_reserve_changes_nothing_where_pages_are_missing():
    b = Both(5, 3, 8)
    b.reserve([16, 16, 8])
    assert b.reserve([1, 17, 9], advance=False) == [0, 0, 2, 0]
    assert b.reserve([0, 113, 121], advance=False) == [0, 0, 0, 2]
    assert b.reserve([1, 16, 8])[2] == 0
    assert b.reserve([15, 0, 0])[2] == 0
    assert b.reserve([1, 0, 0], advance=False)[2] == 1
    assert b.reserve([0, 0, 0]) == [0, 0, 0, 0]


def test_reserve_and_compact_many_pages():
    """More pages than a round of the scan, more requests than waves, prompts of more columns than a wave has lanes."""
    rng = random.Random(5)
    b = Both(9001, 130, 300)
    b.reserve([rng.choice([0, 1, 15, 16, 17, 900, 3000]) for _ in range(130)])
    b.free(rng.sample(range(130), 60))
    b.compact()
    empty = [i for i in range(130) if b.pool.held[i] == 0]
    full = [i for i in range(130) if b.pool.held[i] > 0]
    b.fork([rng.choice(full) for _ in empty], empty)
    b.reserve([rng.choice([0, 1, 1, 40]) for _ in range(130)])
    b.free(rng.sample(range(130), 50))
    b.reserve([rng.choice([0, 1, 1, 40]) if b.pool.held[i] else 0 for i in range(130)])
    b.compact()


@pytest.mark.parametrize("seed", range(6))
def test_random_calls(seed):
    rng = random.Random(seed)
    n, cols, size = rng.randint(1, 12), rng.randint(1, 9), rng.choice([16, 32, 64, 128])
    b = Both(rng.randint(1, 60), n, cols, size)
    for _ in range(25):
        what = rng.randrange(4)
        some = [rng.randrange(-1, n + 1) for _ in range(rng.randint(1, 5))]
        if what == 0:
            b.free(some)
        elif what == 1:
            b.fork(some, [rng.randrange(-1, n + 1) for _ in some])
        elif what == 2:
            b.reserve([rng.choice([0, 0, 1, 5, size, 3 * size]) for _ in range(n)])
        else:
            b.compact()


def test_holes_and_foreign_entries():
    b = Both(10, 3, 4)
    b.load([[3, -1, 7, 99], [7, 3, -4, -1], [-1] * 4], [40, 20, 0])
    b.pool.refs = [0, 0, 0, 2, 0, 0, 0, 2, 0, 0]
    b.pages.refs.copy_(ints(b.pool.refs))
    b.fork([0], [2])
    assert b.pool.table[2] == [3, -1, 7, -1]
    b.compact()
    b.free([0, 1, 2])
    assert b.pool.refs == [0] * 10


def test_compact_elsewhere():
    b = Both(30, 3, 6)
    b.reserve([50, 70, 30])
    b.free([0])
    table, refs = b.pages.page_table.clone(), b.pages.refs.clone()
    out = scd.Pages(torch.full_like(table, 77), torch.full_like(refs, 77), torch.full_like(b.pages.held, 77), 16)
    scd.scd_pages_compact(b.pages, b.moves, out)
    assert torch.equal(b.pages.page_table, table) and torch.equal(b.pages.refs, refs)
    moves, status = b.pool.compact()
    assert out.page_table.tolist() == b.pool.table and out.refs.tolist() == b.pool.refs
    assert (out.held == 77).all() and b.moves.status.tolist() == status


def test_copy_counts_and_sizes():
    """A count beyond the list, negative ones, pages that do not exist, planes of any size."""
    widths = [4, 12, 16, 16384, 16400, 40000, 36]
    planes = [torch.randint(0, 255, (9, w), dtype=torch.uint8, device="cuda") for w in widths]
    lib, pairs = scd.load_library(), ints([[1, 0], [2, 9], [-1, 3], [4, 5], [7, 8]])
    arr = (scd._CPlane * len(planes))(*[scd._CPlane(p.data_ptr(), p.shape[1]) for p in planes])
    for count, done in ((0, []), (-3, []), (1, [(1, 0)]), (4, [(1, 0), (4, 5)]), (1000, [(1, 0), (4, 5), (7, 8)])):
        status = ints([count, 0, 0, 0])
        moves = scd.Moves(pairs, status)
        want = [p.clone() for p in planes]
        for w in want:
            for a, b in done:
                w[b] = w[a]
        assert lib.scd_pages_copy(len(planes), arr, 9, moves._c, torch.cuda.current_stream().cuda_stream) == 0
        for w, p in zip(want, planes):
            assert torch.equal(w, p)


def test_copy_many_layers():
    """More planes than one launch takes."""
    caches = [scd.LatentCache(randn(i, 6, 16, 96).bfloat16(), ints([[0]]), 64) for i in range(300)]
    want = [c.pages.clone() for c in caches]
    scd.scd_pages_copy(caches, scd.Moves(ints([[1, 4], [0, 2]]), ints([2, 0, 0, 0])))
    for w, c in zip(want, caches):
        w[4], w[2] = w[1], w[0]
        assert torch.equal(w, c.pages)


def test_captured():
    """A step of a search in a graph: its lists and lengths change in device memory between replays."""
    b, e = Both(50, 4, 6), Both(50, 4, 6)
    for x in (b, e):
        x.reserve([20, 40, 0, 0])
    src, dst, cu = ints([0, 1]), ints([2, 3]), ints([0, 1, 2, 3, 4])
    batch = scd.Batch(4, cu)
    calls = [scd.prepare_pages_free(b.pages, dst), scd.prepare_pages_fork(b.pages, src, dst),
             scd.prepare_pages_reserve(b.pages, batch, b.moves), scd.prepare_pages_copy(b.caches, b.moves),
             scd.prepare_pages_compact(b.pages, b.moves)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        for call in calls:
            call(side)
    torch.cuda.current_stream().wait_stream(side)
    for s, d in (([0, 1], [2, 3]), ([2, 2], [0, 1]), ([1, 1], [3, 0])):
        src.copy_(ints(s))
        dst.copy_(ints(d))
        g.replay()
        torch.cuda.synchronize()
        e.pool.free(d)
        e.pool.fork(s, d)
        e.pool.reserve([1, 1, 1, 1])
        e.pool.compact()
        assert b.pages.page_table.tolist() == e.pool.table and b.pages.refs.tolist() == e.pool.refs


def test_forked_requests_attend_alike():
    """Both caches behind shared and copied pages: a fork and its source see the same, then their own tokens."""
    size, heads = 16, 4
    n_pages, table = 12, ints([[-1] * 4, [-1] * 4])
    pages = scd.Pages(table, ints([0] * n_pages), ints([0, 0]), size)
    moves = scd.Moves(ints([[0, 0]] * 6), ints([0] * 4))
    lat = scd.LatentCache(torch.zeros(n_pages, size, 96, device="cuda").bfloat16(), table, 64)
    kv = scd.PagedCache(*[torch.zeros(n_pages, 2, size, 32, dtype=torch.int8, device="cuda") for _ in "kv"],
                        *[torch.zeros(n_pages, 2, device="cuda") for _ in "kv"], table)
    w_k, w_v = randn(1, heads, 32, 64).bfloat16() / 8, randn(2, heads, 32, 64).bfloat16() / 8

    def step(new, cu, held, seed):
        batch = scd.Batch(cu[-1], ints(cu), ints(held))
        pages.held.copy_(ints(held))
        scd.scd_pages_reserve(pages, batch, moves)
        scd.scd_pages_copy([lat, kv], moves)
        c, k, v = randn(seed, cu[-1], 96).bfloat16(), randn(seed + 1, cu[-1], 2, 32).bfloat16(), randn(seed + 2, cu[-1], 2, 32).bfloat16()
        if new == "same":
            for x in (c, k, v):
                x[1] = x[0]
        scd.scd_latent_append(lat, batch, c[:, :64], c[:, 64:])
        scd.scd_cache_append(kv, batch, k, v)
        q, p = randn(7, 1, heads, 64).bfloat16().expand(cu[-1], -1, -1).contiguous(), randn(8, 1, heads, 32).bfloat16().expand(cu[-1], -1, -1).contiguous()
        a, o = torch.empty(cu[-1], heads, 32, dtype=torch.bfloat16, device="cuda"), torch.empty_like(p)
        scd.scd_latent_attend(lat, batch, q, w_k, w_v, a)
        scd.scd_cache_attend(kv, batch, p, o)
        return a, o

    step("prompt", [0, 21, 21], [0, 0], 10)
    pages.held.copy_(ints([21, 0]))
    scd.scd_pages_fork(pages, ints([0]), ints([1]))
    assert table[0, :2].tolist() == table[1, :2].tolist()
    for a in step("same", [0, 1, 2], [21, 21], 20):
        assert torch.equal(a[0], a[1]) and a[0].any()
    assert moves.status.tolist()[0] == 1 and table[0, 0] == table[1, 0] and table[0, 1] != table[1, 1]
    for a in step("own", [0, 1, 2], [22, 22], 30):
        assert not torch.equal(a[0], a[1])
