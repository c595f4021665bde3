"""How far attention may be off, value by value, from how errors add up (not from their worst case).

A score is a sum of C products in fp32, rounded at every addition: its error is a walk of C steps of at most half a
step of the partial sums, which are as large as the root of the sum of the products' squares (`norm`).  Errors of
different positions' scores are independent, and so are roundings of different weights: a result sum_j p_j v_j is
off by the root of the sum of the squares of what each position adds, (p_j e_j v_j)^2, and by its own half step.  Every
figure below is an upper estimate of one standard deviation; SIGMAS of them are allowed.
"""
import numpy as np

from oracle import latent_oracle as L

F32 = 2.0 ** -24                      # half a step of fp32, relative to the value
PAIR = 2.0 ** -16                     # two bf16 summands: what the second one's rounding leaves
EXP2 = 2.0 ** -22                     # the exponential
ONCE = 2.0 ** -9                      # one rounding to bf16, at most 2^-8 of the value
SIGMAS = 8.0
MANTISSA = {"bf16": 7, "f32": 23}


def half_step(dtype, x):
    """Half a step of the type at magnitude x."""
    _, e = np.frexp(np.maximum(np.abs(x), 2.0 ** -120))
    return np.ldexp(0.5, e - 1 - MANTISSA[dtype])


def weights_error(dtype, score, norm, channels, inexact_queries, once=False):
    """Standard deviation of a weight's relative error: of its score (sum, scale, difference from the base), of the
    exponential, of its two summands in bf16 (or of its one rounding)."""
    e = F32 * np.sqrt(channels) * norm + 4 * F32 * np.abs(score) + EXP2
    if dtype == "bf16":
        e = e + (ONCE if once else PAIR) + (PAIR * norm if inexact_queries else 0.0)
    return e


def row_error(p, e, v, want):
    """Of sum_j p_j v_j with weights off by e_j, divided by the sum of the same weights."""
    pe = p * e
    return np.sqrt((pe ** 2) @ (v ** 2)) + np.abs(want) * np.sqrt((pe ** 2).sum(1, keepdims=True))


def _products(a, b):
    return np.sqrt((a ** 2) @ (b ** 2))


def over_latents(dtype, rows, seen, q, w_k, w_v, scale):
    """(The definition in 64 bits, what is allowed) of query rows q [n, heads, plain + turned] over cached rows
    [m, latent + turned], of which `seen` [n, m] says which they attend to."""
    h, plain, r = w_k.shape
    out, off = (np.zeros((q.shape[0], h, w_v.shape[1])) for _ in "ab")
    c, t = rows[:, :r], rows[:, r:]
    steps = np.sqrt(rows.shape[0] / 16 + 64)   # additions to a result, joins with them
    for i in range(h):
        x, y = q[:, i, :plain], q[:, i, plain:]
        absorbed, wide = x @ w_k[i], _products(x, w_k[i])
        score = scale * (absorbed @ c.T + y @ t.T)
        norm = np.abs(scale) * np.sqrt((wide ** 2 + absorbed ** 2) @ (c ** 2).T + (y ** 2) @ (t ** 2).T)
        e = weights_error(dtype, score, norm, r + t.shape[1] + plain, True)
        p = L.softmax_rows(score, seen)
        v = c @ w_v[i].T
        want = p @ v
        joined = _products(np.sqrt((p @ c) ** 2 + (p ** 2) @ (c ** 2)), w_v[i].T)
        more = F32 * (steps + np.sqrt(r)) + (PAIR if dtype == "bf16" else 0.0)
        err = SIGMAS * (row_error(p, e, v, want) + more * joined)
        out[:, i], off[:, i] = want, err + half_step(dtype, np.abs(want) + err)
    return out, off


def latent_attend(dtype, pages, table, cu, pos0, q, w_k, w_v, scale):
    """(The definition in 64 bits, what is allowed) of a batch over its pages."""
    out, off = (np.zeros((q.shape[0], w_k.shape[0], w_v.shape[1])) for _ in "ab")
    for b in range(len(cu) - 1):
        n, at = cu[b + 1] - cu[b], slice(cu[b], cu[b + 1])
        if n > 0:
            rows, there = L.rows_held(pages, table, b, 0, max(0, pos0[b] + n))
            seen = there[None] & (np.arange(rows.shape[0])[None] <= (pos0[b] + np.arange(n))[:, None])
            out[at], off[at] = over_latents(dtype, rows, seen, q[at], w_k, w_v, scale)
    return out, off


def rows_attend(dtype, cu, pos0, held_cu, held_pos0, q, k, v, scale, once=False):
    """As latent_attend, over dense rows.  once: weights are rounded to bf16 once."""
    group = q.shape[1] // k.shape[1]
    out, off = (np.zeros((q.shape[0], q.shape[1], v.shape[2])) for _ in "ab")
    for b in range(len(cu) - 1):
        at, rows = slice(cu[b], cu[b + 1]), slice(held_cu[b], held_cu[b + 1])
        n, m = cu[b + 1] - cu[b], held_cu[b + 1] - held_cu[b]
        seen = (held_pos0[b] + np.arange(m))[None] <= (pos0[b] + np.arange(n))[:, None]
        for i in range(q.shape[1]):
            x, y, z = q[at, i], k[rows, i // group], v[rows, i // group]
            score = scale * (x @ y.T)
            e = weights_error(dtype, score, np.abs(scale) * _products(x, y.T), x.shape[1], False, once)
            p = L.softmax_rows(score, seen)
            want = p @ z
            more = F32 * np.sqrt(m / 16 + 64) * np.sqrt(want ** 2 + (p ** 2) @ (z ** 2))
            err = SIGMAS * (row_error(p, e, z, want) + more)
            out[at, i], off[at, i] = want, err + half_step(dtype, np.abs(want) + err)
    return out, off


def assert_close(got, want, off):
    wrong = ~(np.abs(got - want) <= off)
    at = tuple(np.argwhere(wrong)[0]) if wrong.any() else ()
    assert not wrong.any(), (int(wrong.sum()), wrong.size, at, got[at], want[at], off[at])
