"""fp64 oracle of the serving operators: rotary positions, the paged 8-bit cache, attention over it.

Plain numpy, row by row, from the definitions in ``include/scd.h``; it shares no code with the HIP
path.  Rows are [tokens, heads, d]; a batch is (cu, pos0) as lists.  Pages are int8 arrays
[n_pages, heads, page, d] with scales [n_pages, heads].
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(rd, theta, scaling="none", factor=1.0, low=1.0, high=32.0, trained=0):
    base = theta * factor ** (rd / (rd - 2)) if scaling == "ntk" else theta
    out = []
    for i in range(rd // 2):
        w = base ** (-2.0 * i / rd)
        if scaling == "linear":
            w = w / factor
        elif scaling == "by_parts":
            n = trained / (2.0 * math.pi / w)  # trained context over the wavelength
            g = (n - low) / (high - low)
            g = 0.0 if g < 0 else 1.0 if g > 1 else g
            w = (1.0 - g) * (w / factor) + g * w
        out.append(w)
    return np.array(out)


def rotate(x, positions, w, layout="half", gain=1.0, transpose=False):
    """x [tokens, heads, d]; pair i turns by positions * w[i]."""
    y = np.array(x, dtype=np.float64)
    half = len(w)
    for t, p in enumerate(positions):
        for i in range(half):
            a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = gain * math.cos(p * w[i]), gain * math.sin(p * w[i])
            if transpose:
                s = -s
            u, v = y[t, :, a].copy(), y[t, :, b].copy()
            y[t, :, a] = u * c - v * s
            y[t, :, b] = v * c + u * s
    return y


def page_of(table, n_pages, size, b, p):
    if p < 0 or p // size >= table.shape[1]:
        return -1
    page = int(table[b, p // size])
    return page if 0 <= page < n_pages else -1


def append(pages, scales, table, cu, pos0, x):
    """Appends rows x [tokens, heads, d] (fp64, keys turned already); pages (as fp64) and scales are
    updated in place.  Returns x / scale before rounding, per (page, head, slot), for a caller that
    wants to know how near a tie a value was."""
    n_pages, heads, size, d = pages.shape
    ratio = np.full(pages.shape, np.nan)
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        by_page = {}
        for i in range(n):
            page = page_of(table, n_pages, size, b, pos0[b] + i)
            if page >= 0:
                by_page.setdefault(page, []).append(i)
        for page, rows in by_page.items():
            slots = [(pos0[b] + i) % size for i in rows]
            for h in range(heads):
                new = x[[cu[b] + i for i in rows], h]
                old = scales[page, h] if slots[0] > 0 else 0.0
                scale = max(old, np.abs(new).max() / 127.0) if np.isfinite(new).all() else np.nan
                if old != old:
                    scale = np.nan
                if scale < 2.0 ** -126:
                    scale = 0.0
                if scale > old and slots[0] > 0:
                    kept = pages[page, h, :slots[0]] * old / scale
                    ratio[page, h, :slots[0]] = kept
                    pages[page, h, :slots[0]] = np.rint(kept)
                for slot, row in zip(slots, new):
                    r = row / scale if scale > 0 else np.zeros(d)
                    ratio[page, h, slot] = r
                    pages[page, h, slot] = np.clip(np.rint(r), -127, 127)
                scales[page, h] = scale
    return ratio


def attend(q, k_pages, v_pages, k_scales, v_scales, table, cu, pos0, scale):
    """out [tokens, q heads, d], and sum_j p_j |v_j| and the largest scale * sum |q||k| of each row
    (what a tolerance is derived from)."""
    n_pages, heads, size, d = k_pages.shape
    group = q.shape[1] // heads
    out, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        seen, ids = [], []
        for j in range(pos0[b] + n):
            page = page_of(table, n_pages, size, b, j)
            if page >= 0:
                seen.append(j)
                ids.append(page)
        seen, ids = np.array(seen, dtype=np.int64), np.array(ids, dtype=np.int64)
        for h in range(heads):
            k = k_pages[ids, h, seen % size].astype(np.float64) * k_scales[ids, h].astype(np.float64)[:, None]
            v = v_pages[ids, h, seen % size].astype(np.float64) * v_scales[ids, h].astype(np.float64)[:, None]
            for i in range(n):
                m = int(np.searchsorted(seen, pos0[b] + i, side="right"))
                if m == 0:
                    continue
                for g in range(h * group, (h + 1) * group):
                    row = q[cu[b] + i, g]
                    s = scale * (k[:m] @ row)
                    p = np.exp(s - s.max())
                    p = p / p.sum()
                    out[cu[b] + i, g] = p @ v[:m]
                    mass[cu[b] + i, g] = p @ np.abs(v[:m])
                    reach[cu[b] + i, g] = abs(scale) * (np.abs(k[:m]) @ np.abs(row)).max()
    return out, mass, reach
