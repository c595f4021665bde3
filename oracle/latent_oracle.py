"""fp64 oracle of the latent cache, of attention over it and over dense rows, and of the pages' bookkeeping.

Plain numpy, row by row, and plain lists, from the definitions in ``include/scd.h``; it shares no code
with the HIP path.  Cached rows are [n_pages, page, latent + turned]; a batch is (cu, pos0) as lists.
"""
from __future__ import annotations

import numpy as np

from .serving_oracle import page_of, rotate


def append(pages, table, cu, pos0, latent, turned, w=None, layout="half", gain=1.0):
    """Rows into the pages, in place; w: frequencies of the shared key's pairs (None: as it is)."""
    n_pages, size, _ = pages.shape
    for b in range(len(cu) - 1):
        for i in range(cu[b + 1] - cu[b]):
            t, p = cu[b] + i, pos0[b] + i
            page = page_of(table, n_pages, size, b, p)
            if page < 0:
                continue
            key = turned[t][None, None]
            if w is not None:
                key = rotate(key, [p], w, layout, gain)
            pages[page, p % size] = np.concatenate([latent[t], key[0, 0]])


def rows_held(pages, table, b, first, n):
    """Rows of positions first .. first + n - 1 of request b, and which of them are there."""
    n_pages, size, width = pages.shape
    rows, there = np.zeros((n, width)), np.zeros(n, dtype=bool)
    for i in range(n):
        page = page_of(table, n_pages, size, b, first + i)
        if page >= 0:
            rows[i], there[i] = pages[page, (first + i) % size], True
    return rows, there


def expand(pages, table, cu, pos0, w_k, w_v):
    h, plain, r = w_k.shape
    k = np.zeros((cu[-1], h, plain + pages.shape[2] - r))
    v = np.zeros((cu[-1], h, w_v.shape[1]))
    for b in range(len(cu) - 1):
        rows, _ = rows_held(pages, table, b, pos0[b], cu[b + 1] - cu[b])
        at = slice(cu[b], cu[b + 1])
        k[at, :, :plain] = np.einsum("tr,hdr->thd", rows[:, :r], w_k)
        k[at, :, plain:] = rows[:, None, r:]
        v[at] = np.einsum("tr,hdr->thd", rows[:, :r], w_v)
    return k, v


def softmax_rows(score, seen):
    """softmax over the positions that a row sees; zeros for a row that sees none."""
    score = np.where(seen, score, -np.inf)
    top = score.max(-1, keepdims=True, initial=-np.inf)
    e = np.where(seen, np.exp(score - np.where(np.isneginf(top), 0.0, top)), 0.0)
    total = e.sum(-1, keepdims=True)
    return np.divide(e, total, out=np.zeros_like(e), where=total != 0)


def latent_attend(pages, table, cu, pos0, q, w_k, w_v, scale):
    """Every head's own keys and values, and a bound on what each result's terms add up to: (out, the sum of
    p_j |w| |c_j|, the largest score's sum of magnitudes)."""
    h, plain, r = w_k.shape
    out, mass, loud = (np.zeros((q.shape[0], h, w_v.shape[1])) for _ in range(3))
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        rows, there = rows_held(pages, table, b, 0, max(0, pos0[b] + n))
        seen = there[None] & (np.arange(rows.shape[0])[None] <= (pos0[b] + np.arange(n))[:, None])
        c, t = rows[:, :r], rows[:, r:]
        for i in range(h):
            x = q[cu[b]:cu[b + 1], i]
            score = scale * (x[:, :plain] @ (c @ w_k[i].T).T + x[:, plain:] @ t.T)
            p = softmax_rows(score, seen)
            out[cu[b]:cu[b + 1], i] = p @ (c @ w_v[i].T)
            mass[cu[b]:cu[b + 1], i] = (p @ np.abs(c)) @ np.abs(w_v[i]).T
            parts = np.abs(scale) * (np.abs(x[:, :plain]) @ np.abs(w_k[i]) @ np.abs(c).T + np.abs(x[:, plain:]) @ np.abs(t).T)
            loud[cu[b]:cu[b + 1], i] = np.where(seen, parts, 0).max(1, initial=0)[:, None]
    return out, mass, loud


def rows_attend(cu, pos0, held_cu, held_pos0, q, k, v, scale):
    """As latent_attend, over dense rows."""
    group = q.shape[1] // k.shape[1]
    out, mass, loud = (np.zeros((q.shape[0], q.shape[1], v.shape[2])) for _ in range(3))
    for b in range(len(cu) - 1):
        at, rows = slice(cu[b], cu[b + 1]), slice(held_cu[b], held_cu[b + 1])
        n, m = cu[b + 1] - cu[b], held_cu[b + 1] - held_cu[b]
        seen = (held_pos0[b] + np.arange(m))[None] <= (pos0[b] + np.arange(n))[:, None]
        for i in range(q.shape[1]):
            x, y, z = q[at, i], k[rows, i // group], v[rows, i // group]
            p = softmax_rows(scale * (x @ y.T), seen)
            out[at, i] = p @ z
            mass[at, i] = p @ np.abs(z)
            loud[at, i] = np.where(seen, np.abs(scale) * (np.abs(x) @ np.abs(y).T), 0).max(1, initial=0)[:, None]
    return out, mass, loud


# ---- pages -----------------------------------------------------------------------------------------------
class Pool:
    """The bookkeeping as lists, one request and one page after another."""

    def __init__(self, table, refs, held, size):
        self.table, self.refs, self.held, self.size = [list(r) for r in table], list(refs), list(held), size

    def names(self, p):
        return 0 <= p < len(self.refs)

    def free(self, seqs):
        for b in dict.fromkeys(seqs):
            if not 0 <= b < len(self.table):
                continue
            for p in self.table[b]:
                if self.names(p):
                    self.refs[p] = max(0, self.refs[p] - 1)
            self.table[b] = [-1] * len(self.table[b])
            self.held[b] = 0

    def fork(self, src, dst):
        n = len(self.table)
        empty = [h == 0 and not any(self.names(p) for p in row) for h, row in zip(self.held, self.table)]
        for i, (a, d) in enumerate(zip(src, dst)):
            if not (0 <= a < n and 0 <= d < n) or not empty[d] or d in dst[:i] or a in dst:
                continue
            for j, p in enumerate(self.table[a]):
                keep = self.names(p) and j * self.size < self.held[a]
                self.table[d][j] = p if keep else -1
                if keep:
                    self.refs[p] += 1
            self.held[d] = self.held[a]

    def reserve(self, new):
        """(moves, status): nothing changes where status[2] or status[3] is set."""
        before = [list(r) for r in self.table], list(self.refs)
        wrong = sum(n > 0 and (h < 0 or h + n > len(row) * self.size)
                    for n, h, row in zip(new, self.held, self.table))
        if wrong:
            return [], [0, 0, 0, wrong]
        free = [p for p, n in enumerate(self.refs) if n <= 0]
        moves, taken = [], 0
        for b, n in enumerate(new):
            if n <= 0:
                continue
            for j in range(self.held[b] // self.size, -(-(self.held[b] + n) // self.size)):
                p = self.table[b][j]
                if self.names(p) and self.refs[p] <= 1:
                    continue
                taken += 1
                if taken > len(free):
                    if self.names(p):
                        self.refs[p] -= 1
                    continue
                fresh = free[taken - 1]
                self.table[b][j], self.refs[fresh] = fresh, 1
                if self.names(p):
                    self.refs[p] -= 1
                    if j * self.size < self.held[b]:
                        moves.append((p, fresh))
        if taken > len(free):
            self.table, self.refs = before
            return [], [0, 0, taken - len(free), 0]
        return moves, [len(moves), 0, 0, 0]

    def compact(self):
        used = sum(n > 0 for n in self.refs)
        gaps = [p for p in range(used) if self.refs[p] <= 0]
        high = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(high, gaps))
        self.table = [[to.get(p, p) if self.names(p) else -1 for p in row] for row in self.table]
        counts = [max(0, n) for n in self.refs]
        for a, b in to.items():
            counts[a], counts[b] = 0, counts[a]
        self.refs = counts
        return list(zip(high, gaps)), [len(high), used, 0, 0]
