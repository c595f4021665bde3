"""Pins of the oracle of the latent cache and of the pages: against each other, closed forms and invariants (CPU)."""
import random

import numpy as np
import pytest

from oracle import latent_oracle as L


def _cache(rng, lens, size, width, holes=()):
    need = [-(-n // size) for n in lens]
    order = rng.permutation(sum(need) + 2).tolist()
    table = np.full((len(lens), max(need)), -1)
    for b, n in enumerate(need):
        table[b, :n] = [order.pop() for _ in range(n)]
    for b, j in holes:
        table[b, j] = -1
    return rng.standard_normal((sum(need) + 2, size, width)), table


@pytest.mark.parametrize("holes", [(), ((0, 1),), ((1, 0), (0, 2))])
def test_absorbed_is_expanded_attention(holes):
    """Attention over the latents equals attention over every head's own keys and values, holes left out."""
    rng = np.random.default_rng(1)
    lens, held, r, dr, h = [3, 2], [9, 5], 6, 4, 3
    pages, table = _cache(rng, [12, 7], 4, r + dr, holes)
    w_k, w_v = rng.standard_normal((h, 5, r)), rng.standard_normal((h, 7, r))
    q = rng.standard_normal((5, h, 5 + dr))
    cu = [0, 3, 5]
    got, mass, loud = L.latent_attend(pages, table, cu, held, q, w_k, w_v, 0.4)
    for b in range(2):
        total = held[b] + lens[b]
        rows, there = L.rows_held(pages, table, b, 0, total)
        k, v = L.expand(pages, table[b:b + 1], [0, total], [0], w_k, w_v)
        for i in range(lens[b]):
            see = [j for j in range(total) if there[j] and j <= held[b] + i]
            for a in range(h):
                s = np.array([0.4 * q[cu[b] + i, a] @ k[j, a] for j in see])
                p = np.exp(s) / np.exp(s).sum()
                assert np.allclose(got[cu[b] + i, a], sum(x * v[j, a] for x, j in zip(p, see)), rtol=0, atol=1e-12)
    assert np.all(np.abs(got) <= mass + 1e-12) and np.all(loud >= 0)


def test_rows_attend_closed_forms():
    """Equal keys average the values seen; one loud key picks its value; grouped heads read their own rows; in front of
    all rows nothing is seen."""
    v = np.arange(12.0).reshape(6, 2, 1)
    same = L.rows_attend([0, 3], [3], [0, 6], [0], np.ones((3, 4, 2)), np.ones((6, 2, 2)), v, 1.0)[0]
    for i in range(3):
        for h in range(4):
            assert np.isclose(same[i, h, 0], v[:4 + i, h // 2, 0].mean())
    k = np.zeros((6, 2, 2))
    k[2, :, 0] = 1.0
    loud = L.rows_attend([0, 1], [5], [0, 6], [0], np.ones((1, 2, 2)), k, v, 60.0)[0]
    assert np.allclose(loud[0, :, 0], v[2, :, 0])
    assert not L.rows_attend([0, 2], [0], [0, 6], [2], np.ones((2, 2, 2)), k, v, 1.0)[0].any()


def test_append_then_held():
    rng = np.random.default_rng(2)
    pages, table = _cache(rng, [10], 4, 6)
    c, t = rng.standard_normal((3, 4)), rng.standard_normal((3, 2))
    L.append(pages, table, [0, 3], [5], c, t, np.array([0.3]))
    rows, there = L.rows_held(pages, table, 0, 5, 3)
    assert there.all() and np.array_equal(rows[:, :4], c)
    for i, p in enumerate((5, 6, 7)):
        z = complex(*t[i]) * np.exp(0.3j * p)
        assert np.allclose(rows[i, 4:], [z.real, z.imag])


@pytest.mark.parametrize("seed", range(20))
def test_pool_invariants(seed):
    """Counts are the entries that name a page, what requests hold follows them through every call, and a page that a
    request writes to is its own."""
    rng = random.Random(seed)
    n, cols, size = rng.randint(1, 6), rng.randint(1, 6), 4
    pool = L.Pool([[-1] * cols for _ in range(n)], [0] * rng.randint(1, 20), [0] * n, size)
    text = {}       # page -> the tokens in it
    story = [[] for _ in range(n)]

    def check():
        for p, refs in enumerate(pool.refs):
            assert refs == sum(p == q for row in pool.table for q in row)
        for b in range(n):
            assert [text[pool.table[b][i // size]][i % size] for i in range(pool.held[b])] == story[b]

    for step in range(40):
        what = rng.randrange(4)
        if what == 0:
            gone = [rng.randrange(n) for _ in range(rng.randint(0, 2))]
            pool.free(gone)
            for b in gone:
                story[b] = []
        elif what == 1:
            src, dst = rng.randrange(n), rng.randrange(n)
            empty = pool.held[dst] == 0 and src != dst and all(p < 0 for p in pool.table[dst])
            pool.fork([src], [dst])
            if empty:
                story[dst] = list(story[src])
        elif what == 2:
            new = [rng.choice([0, 1, 3, 5]) for _ in range(n)]
            moves, status = pool.reserve(new)
            for a, b in moves:
                text[b] = list(text[a])
            if not status[2] and not status[3]:
                for b in range(n):
                    for _ in range(new[b]):
                        p = pool.table[b][pool.held[b] // size]
                        assert pool.refs[p] == 1
                        text.setdefault(p, [None] * size)[pool.held[b] % size] = (step, b)
                        story[b].append((step, b))
                        pool.held[b] += 1
        else:
            moves, status = pool.compact()
            for a, b in moves:
                text[b] = text.pop(a, [None] * size)
            assert all(r > 0 for r in pool.refs[:status[1]]) and not any(pool.refs[status[1]:])
        check()
