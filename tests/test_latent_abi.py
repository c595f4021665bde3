"""Refusals of the latent cache's, the dense rows' and the pages' entry points, before anything is launched (CPU)."""
import ctypes

import pytest

import paper_2606_07684_amd as scd

NULL, SHAPE, ALIGN, UNSUP, WORKSPACE = 1, 2, 4, 5, 6
FAKE = 1 << 20  # a device address that no call reaches


@pytest.fixture(scope="module")
def lib():
    return scd.load_library()


def _cache(**kw):
    c = dict(n_pages=10, page_tokens=16, latent_dim=64, turned_dim=32, max_pages=4, pages=FAKE, page_table=FAKE)
    c.update(kw)
    return scd._CLatentCache(**c)


def _batch(n_tokens=5, n_seqs=1, cu=None):
    return scd._CBatch(n_seqs, n_tokens, cu, None)


def _rows(heads=1, token=4096, head=96, data=FAKE):
    return scd._CRows(data, heads, token, head)


def _ref(x):
    return None if x is None else ctypes.byref(x)


BAD_CACHES = [(None, NULL), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(latent_dim=0), UNSUP),
              (dict(latent_dim=48), UNSUP), (dict(latent_dim=544), UNSUP), (dict(turned_dim=0), UNSUP),
              (dict(turned_dim=128), UNSUP), (dict(page_tokens=8), UNSUP), (dict(page_tokens=48), UNSUP),
              (dict(pages=None), NULL), (dict(pages=FAKE + 8), ALIGN), (dict(page_table=None), NULL),
              (dict(page_table=FAKE + 2), ALIGN)]


def test_latent_append(lib):
    def call(cache=_cache(), batch=_batch(), dtype=1, c=_rows(), k=_rows(), rotary=None, table=FAKE, maxp=100):
        return lib.scd_latent_append(_ref(cache), _ref(batch), dtype, _ref(c), _ref(k), _ref(rotary), table, maxp, None)

    for bad, want in BAD_CACHES:
        assert call(cache=None if bad is None else _cache(**bad)) == want, bad
    assert call(batch=None) == NULL
    assert call(batch=_batch(n_seqs=0)) == SHAPE
    assert call(batch=_batch(n_tokens=-1)) == SHAPE
    assert call(batch=_batch(n_seqs=2)) == NULL
    assert call(dtype=2) == SHAPE
    for name in "ck":
        assert call(**{name: None}) == NULL
        assert call(**{name: _rows(data=None)}) == NULL
        assert call(**{name: _rows(heads=2)}) == SHAPE
        assert call(**{name: _rows(data=FAKE + 1)}) == ALIGN
        assert call(**{name: _rows(token=-1)}) == SHAPE
    turns = lambda **kw: scd.Rotary(**dict(dict(head_dim=32, theta=1e4), **kw))._c  # noqa: E731
    assert call(rotary=turns(head_dim=64)) == SHAPE
    assert call(rotary=turns(), table=None) == WORKSPACE
    assert call(rotary=turns(), table=FAKE + 8) == ALIGN
    assert call(rotary=turns(), maxp=0) == WORKSPACE
    assert call(rotary=turns(theta=0.5)) == SHAPE
    assert call(batch=_batch(n_tokens=0), c=_rows(data=None), k=_rows(data=None)) == 0


def test_latent_attend(lib):
    def call(cache=_cache(), batch=_batch(), dtype=1, scale=0.1, plain=64, value=64, w_k=FAKE, w_v=FAKE,
             q=_rows(4), out=_rows(4), ws=FAKE, nbytes=1 << 40):
        return lib.scd_latent_attend(_ref(cache), _ref(batch), dtype, scale, plain, value, w_k, w_v, _ref(q), _ref(out),
                                     ws, nbytes, None)

    for bad, want in BAD_CACHES:
        assert call(cache=None if bad is None else _cache(**bad)) == want, bad
    assert call(batch=None) == NULL
    assert call(dtype=-1) == SHAPE
    for s in (float("nan"), float("inf"), 1e39):
        assert call(scale=s) == SHAPE
    for bad in (0, 16, 100, 288):
        assert call(plain=bad) == UNSUP and call(value=bad) == UNSUP
    assert call(w_k=None) == NULL and call(w_v=None) == NULL
    assert call(w_k=FAKE + 8) == ALIGN and call(w_v=FAKE + 8) == ALIGN
    assert call(q=None) == NULL and call(out=None) == NULL
    assert call(q=_rows(0)) == SHAPE and call(out=_rows(3)) == SHAPE
    assert call(q=_rows(data=FAKE + 1)) == ALIGN
    assert call(out=_rows(4, head=63)) == SHAPE                       # heads overlap
    assert call(out=_rows(4, token=100)) == SHAPE
    assert call(q=_rows(65536)) == UNSUP
    assert call(batch=_batch(n_tokens=65536)) == UNSUP
    assert call(batch=_batch(n_tokens=60000), q=_rows(4096), out=_rows(4096)) == UNSUP
    need = lib.scd_latent_attend_workspace_bytes(_ref(_cache()), _ref(_batch()), 1, 4)
    assert need > 0
    assert call(ws=None) == NULL and call(ws=FAKE + 8) == ALIGN and call(nbytes=need - 1) == SHAPE
    assert call(batch=_batch(n_tokens=0), q=_rows(4, data=None), out=_rows(4, data=None), ws=None, nbytes=0) == 0
    size = lib.scd_latent_attend_workspace_bytes
    assert size(None, _ref(_batch()), 1, 4) == size(_ref(_cache()), None, 1, 4) == 0
    assert size(_ref(_cache()), _ref(_batch()), 3, 4) == size(_ref(_cache()), _ref(_batch()), 1, 0) == 0
    assert size(_ref(_cache()), _ref(_batch(n_tokens=0)), 1, 4) == 0


def test_latent_expand(lib):
    def call(cache=_cache(), batch=_batch(), dtype=1, heads=4, plain=64, value=64, w_k=FAKE, w_v=FAKE, k=_rows(4),
             v=_rows(4)):
        return lib.scd_latent_expand(_ref(cache), _ref(batch), dtype, heads, plain, value, w_k, w_v, _ref(k), _ref(v), None)

    for bad, want in BAD_CACHES:
        assert call(cache=None if bad is None else _cache(**bad)) == want, bad
    assert call(batch=None) == NULL and call(dtype=7) == SHAPE
    assert call(heads=0) == SHAPE and call(heads=65536) == UNSUP
    assert call(plain=48) == UNSUP and call(value=300) == UNSUP
    assert call(w_k=None) == NULL and call(w_v=FAKE + 4) == ALIGN
    assert call(k=None) == NULL and call(v=None) == NULL
    assert call(k=_rows(3)) == SHAPE and call(v=_rows(5)) == SHAPE
    assert call(k=_rows(4, head=95)) == SHAPE                          # 64 + 32 channels
    assert call(v=_rows(4, head=0)) == SHAPE
    assert call(batch=_batch(n_tokens=0), k=_rows(4, data=None), v=_rows(4, data=None)) == 0


def test_rows_attend(lib):
    def call(batch=_batch(), held=_batch(9), dtype=1, scale=0.1, key=64, value=64, q=_rows(4), k=_rows(2), v=_rows(2),
             out=_rows(4), ws=FAKE, nbytes=1 << 40):
        return lib.scd_rows_attend(_ref(batch), _ref(held), dtype, scale, key, value, _ref(q), _ref(k), _ref(v), _ref(out),
                                   ws, nbytes, None)

    assert call(batch=None) == NULL and call(held=None) == NULL
    assert call(held=_batch(9, 2, FAKE)) == SHAPE
    assert call(dtype=2) == SHAPE and call(scale=float("nan")) == SHAPE
    for bad in (0, 16, 200, 224):
        assert call(key=bad) == UNSUP
    for bad in (0, 40, 160):
        assert call(value=bad) == UNSUP
    for name in ("q", "k", "v", "out"):
        assert call(**{name: None}) == NULL
        assert call(**{name: _rows({"q": 4, "out": 4}.get(name, 2), data=None)}) == NULL
        assert call(**{name: _rows({"q": 4, "out": 4}.get(name, 2), data=FAKE + 1)}) == ALIGN
    assert call(k=_rows(3), v=_rows(3)) == SHAPE and call(v=_rows(1)) == SHAPE and call(out=_rows(2)) == SHAPE
    assert call(q=_rows(0)) == SHAPE and call(k=_rows(0)) == SHAPE
    assert call(out=_rows(4, head=32)) == SHAPE
    assert call(q=_rows(65536), out=_rows(65536)) == UNSUP
    many = _batch(1 << 30)
    assert call(batch=many, q=_rows(4, token=400), out=_rows(4, token=400)) == UNSUP
    need = lib.scd_rows_attend_workspace_bytes(_ref(_batch()), _ref(_batch(9999)), 1, 4, 2, 64, 64)
    assert need > 0
    held = _batch(9999)
    assert call(held=held, ws=None) == NULL and call(held=held, ws=FAKE + 4) == ALIGN
    assert call(held=held, nbytes=need - 1) == SHAPE
    assert call(batch=_batch(0), q=_rows(4, data=None), out=_rows(4, data=None)) == 0
    size = lib.scd_rows_attend_workspace_bytes
    assert size(None, _ref(held), 1, 4, 2, 64, 64) == size(_ref(_batch()), None, 1, 4, 2, 64, 64) == 0
    assert size(_ref(_batch()), _ref(held), 1, 4, 3, 64, 64) == size(_ref(_batch()), _ref(held), 1, 4, 0, 64, 64) == 0


def _pages(**kw):
    p = dict(n_pages=10, n_seqs=3, max_pages=4, page_tokens=16, refs=FAKE, page_table=FAKE, held=FAKE)
    p.update(kw)
    return scd._CPages(**p)


def _moves(capacity=10, pairs=FAKE, status=FAKE):
    return scd._CMoves(capacity, pairs, status)


BAD_POOLS = [(None, NULL), (dict(n_pages=0), SHAPE), (dict(n_seqs=0), SHAPE), (dict(max_pages=0), SHAPE),
             (dict(page_tokens=0), SHAPE), (dict(refs=None), NULL), (dict(page_table=None), NULL), (dict(held=None), NULL),
             (dict(refs=FAKE + 1), ALIGN), (dict(page_table=FAKE + 2), ALIGN), (dict(held=FAKE + 3), ALIGN)]


def test_pages_free_and_fork(lib):
    for bad, want in BAD_POOLS:
        pool = None if bad is None else _pages(**bad)
        assert lib.scd_pages_free(_ref(pool), 1, FAKE, None) == want, bad
        assert lib.scd_pages_fork(_ref(pool), 1, FAKE, FAKE, None) == want, bad
        assert lib.scd_pages_workspace_bytes(_ref(pool)) == 0
    pool = _ref(_pages())
    assert lib.scd_pages_free(pool, -1, FAKE, None) == SHAPE and lib.scd_pages_free(pool, 1, None, None) == NULL
    assert lib.scd_pages_free(pool, 1, FAKE + 2, None) == ALIGN and lib.scd_pages_free(pool, 0, None, None) == 0
    assert lib.scd_pages_fork(pool, 1, None, FAKE, None) == NULL and lib.scd_pages_fork(pool, 1, FAKE, None, None) == NULL
    assert lib.scd_pages_fork(pool, -2, FAKE, FAKE, None) == SHAPE and lib.scd_pages_fork(pool, 0, None, None, None) == 0
    assert lib.scd_pages_fork(pool, 1, FAKE + 1, FAKE, None) == ALIGN


def test_pages_reserve_and_compact(lib):
    batch = _batch(5, 3, FAKE)
    need = lib.scd_pages_workspace_bytes(_ref(_pages()))
    assert need > 0

    def reserve(pool=_pages(), b=batch, m=_moves(), ws=FAKE, nbytes=need):
        return lib.scd_pages_reserve(_ref(pool), _ref(b), _ref(m), ws, nbytes, None)

    def compact(pool=_pages(), out=None, m=_moves(), ws=FAKE, nbytes=need):
        return lib.scd_pages_compact(_ref(pool), _ref(out), _ref(m), ws, nbytes, None)

    for bad, want in BAD_POOLS:
        pool = None if bad is None else _pages(**bad)
        assert reserve(pool) == want and compact(pool) == want, bad
        if bad is not None:
            assert compact(out=pool) == want, bad
    assert reserve(b=None) == NULL and reserve(b=_batch(5)) == SHAPE
    for call in (reserve, compact):
        assert call(m=None) == NULL and call(m=_moves(pairs=None)) == NULL and call(m=_moves(status=None)) == NULL
        assert call(m=_moves(pairs=FAKE + 2)) == ALIGN and call(m=_moves(status=FAKE + 1)) == ALIGN
        assert call(ws=None) == NULL and call(ws=FAKE + 8) == ALIGN and call(nbytes=need - 1) == SHAPE
    assert reserve(m=_moves(2)) == SHAPE and compact(m=_moves(4)) == SHAPE
    for other in (dict(n_pages=11), dict(n_seqs=2), dict(max_pages=5), dict(page_tokens=32)):
        assert compact(out=_pages(**other)) == SHAPE


def test_pages_copy(lib):
    def call(planes=((FAKE, 64),), n_pages=10, m=_moves(), n=None):
        arr = None if planes is None else (scd._CPlane * max(1, len(planes)))(*[scd._CPlane(*p) for p in planes])
        return lib.scd_pages_copy(len(planes) if n is None else n, arr, n_pages, _ref(m), None)

    assert call(n=-1) == SHAPE and call(planes=None, n=1) == NULL and call(n_pages=0) == SHAPE
    assert call(m=None) == NULL and call(m=_moves(-1)) == SHAPE and call(m=_moves(status=None)) == NULL
    assert call(((None, 64),)) == NULL and call(((FAKE + 8, 64),)) == ALIGN
    for size in (0, 2, 30, -4, (1 << 30) + 4):
        assert call(((FAKE, 64), (FAKE, size))) == SHAPE
    assert call(((FAKE, 64),), m=_moves(0, None)) == 0


def test_binding_refuses_before_the_library():
    import torch

    cpu = torch.zeros(4, 16, 96)
    with pytest.raises(ValueError, match="CUDA"):
        scd.LatentCache(cpu, torch.zeros(1, 4, dtype=torch.int32), 64)
    with pytest.raises(ValueError, match="page_table"):
        scd.Pages(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2), torch.zeros(2), 16)
    with pytest.raises(ValueError, match="pairs"):
        scd.Moves(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="one cache"):
        scd.prepare_pages_copy([], None)
