"""The serving operators beside the codec as cases that a timing or comparison program can run.

The consumer's cache, once the codec has rebuilt it, is used: queries and keys are rotated to their
positions, keys and values go into a paged cache of 8-bit values with one scale for each page and
head, the cache is read back where dense keys and values are wanted, and new tokens attend to it.
Kinds of pass:
  rotary   queries and keys of packed requests turned to their positions (or, transposed, the
           gradient of that), out of a fused projection's rows
  cache    keys and values appended to the paged 8-bit cache (keys turned on the way where
           ``rotate``), then everything the requests hold read back as dense rows
  attend   new tokens' queries over the paged 8-bit cache, causal, grouped heads

``run`` with ``own`` false computes the same in elementary torch operations in 32 bits; with ``own``
true it calls the framework's entry points.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(dtype="bf16", q_heads=32, kv_heads=8, head_dim=128, page=64, theta=5e5,
                 seqs=1, new=1, ragged=False, held_lo=0, held_hi=0, split=1,
                 rotate=True, rotary_dim=0, layout="half", transpose=False,
                 scaling="none", factor=1.0, trained=0, attention_factor=1.0)


def _case(name, kind, **kw):
    c = dict(_DEFAULTS, kind=kind)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One generated token of each of 16 requests: the smallest call, launch latency decides.
        _case("rotary_token", "rotary", seqs=16, new=16, held_lo=100, held_hi=8000),
        # One 8192-token prompt at the 8B shape, frequencies scaled by parts for a long context.
        _case("rotary_prompt", "rotary", new=8192, scaling="by_parts", factor=8.0, trained=8192),
        # Interleaved pairs in half of a 64-channel head, ragged requests, fp32: the gradient.
        _case("rotary_gradient_f32", "rotary", dtype="f32", q_heads=8, kv_heads=4, head_dim=64,
              theta=1e4, seqs=5, new=10007, ragged=True, rotary_dim=32, layout="interleaved",
              transpose=True),
        # One generated token of each of 64 requests goes into short caches; read back whole.
        _case("cache_token", "cache", seqs=64, new=64, held_lo=1, held_hi=200),
        # The smallest model's 512-token prompt in fp32, pages of 16 tokens.
        _case("cache_tiny_f32", "cache", dtype="f32", q_heads=8, kv_heads=4, head_dim=64, page=16,
              theta=1e4, new=512),
        # One 8192-token prompt at the 8B shape, keys rotated on the way.
        _case("cache_prompt", "cache", new=8192),
        # 16 decoded prefixes of 1K to 16K tokens (keys already rotated) become paged caches.
        _case("cache_import_ragged", "cache", seqs=16, new=111169, ragged=True, rotate=False),
        # One token of one short request: latency decides.
        _case("attend_token_short", "attend", held_lo=332, held_hi=332),
        # One token of each of 16 requests with 1K to 16K tokens: the bulk of generation.
        _case("attend_token_batch", "attend", seqs=16, new=16, held_lo=1023, held_hi=16383),
        # One token of one long request, 28 query heads over 4: few rows, a long axis.
        _case("attend_token_long", "attend", q_heads=28, kv_heads=4, theta=1e6, held_lo=32767,
              held_hi=32767),
        # A few proposed tokens of each of 8 requests, fp32, the smallest model's heads.
        _case("attend_few_f32", "attend", dtype="f32", q_heads=8, kv_heads=4, head_dim=64, page=16,
              theta=1e4, seqs=8, new=37, ragged=True, held_lo=50, held_hi=1500),
        # The last 2048 tokens of an 8192-token prompt over the cache that holds all of it.
        _case("attend_prompt", "attend", new=2048, held_lo=6144, held_hi=6144),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotary", "cache", "attend", "attend"])
    q_heads, kv_heads, head_dim, theta = rng.choice(
        [(32, 8, 128, 5e5), (28, 4, 128, 1e6), (64, 8, 128, 5e5), (8, 4, 64, 1e4), (16, 16, 64, 1e4),
         (8, 2, 32, 1e4)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = _case(None, kind, dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
              theta=theta, page=rng.choice([16, 32, 64, 128]), split=rng.randrange(1 << 20))
    if kind == "rotary":
        new = _between(rng, 1, 8192)
        seqs = min(new, _between(rng, 1, 64))
        c.update(seqs=seqs, new=new, ragged=rng.random() < 0.7, held_hi=rng.randrange(4000),
                 layout=rng.choice(["half", "interleaved"]), transpose=rng.random() < 0.3,
                 rotary_dim=rng.choice([0, 0, head_dim // 2]))
        if rng.random() < 0.5:
            c.update(scaling=rng.choice(["linear", "ntk", "by_parts"]), factor=rng.choice([2.0, 8.0]),
                     trained=4096, attention_factor=rng.choice([1.0, 1.1]))
    elif kind == "cache":
        new = _between(rng, 1, 30000) if dtype == "bf16" else _between(rng, 1, 1000)
        seqs = min(new, _between(rng, 1, 64))
        c.update(seqs=seqs, new=new, ragged=rng.random() < 0.7, held_hi=rng.randrange(300),
                 rotate=rng.random() < 0.6, layout=rng.choice(["half", "interleaved"]))
    elif rng.random() < 0.6:  # a token, or a few, of each request
        seqs = _between(rng, 1, 64)
        held = _between(rng, 32, min(32000, 250000 // seqs))
        c.update(seqs=seqs, new=seqs * rng.choice([1, 1, 1, 2, 5]), ragged=rng.random() < 0.5,
                 held_lo=held // 8, held_hi=held)
    else:  # prompts, some behind a prefix
        new = _between(rng, 16, 1500)
        seqs = rng.choice([1, 1, 2, 3])
        c.update(seqs=seqs, new=new, ragged=rng.random() < 0.7, held_hi=rng.randrange(5000))
    return c


# ---- sizes -------------------------------------------------------------------------------------
def _lengths(c):
    """New tokens and held tokens of every request."""
    rng = random.Random(c["split"])
    n, total = c["seqs"], c["new"]
    if c["ragged"]:
        weight = [rng.uniform(0.1, 1.0) for _ in range(n)]
        new = [int(total * w / sum(weight)) for w in weight]
    else:
        new = [total // n] * n
    new[-1] += total - sum(new)
    return new, [rng.randint(c["held_lo"], c["held_hi"]) for _ in range(n)]


def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def work(case):
    c = dict(_DEFAULTS, **case)
    new, held = _lengths(c)
    eb = 2 if c["dtype"] == "bf16" else 4
    d, hq, hk, t = c["head_dim"], c["q_heads"], c["kv_heads"], sum(new)
    if c["kind"] == "rotary":
        return {"bytes": 2 * t * (hq + hk) * d * eb, "flops": 3 * t * (hq + hk) * (c["rotary_dim"] or d)}
    kv = sum(n + m for n, m in zip(new, held))
    pages = sum(-(-(n + m) // c["page"]) for n, m in zip(new, held))
    if c["kind"] == "cache":
        # the new rows read and stored in 8 bits; everything held read in 8 bits and written dense
        return {"bytes": 2 * hk * (d * (t * (eb + 1) + kv * (1 + eb)) + 8 * pages),
                "flops": 2 * hk * d * (4 * t + kv) + (3 * t * hk * d if c["rotate"] else 0)}
    pairs = sum(n * m + n * (n + 1) // 2 for n, m in zip(new, held))
    return {"bytes": 2 * hk * (kv * d + 4 * pages) + 2 * t * hq * d * eb,
            "flops": 4.0 * d * hq * pairs}


# ---- inputs ------------------------------------------------------------------------------------
def _frequencies(c):
    """Radians a position turns each channel pair by."""
    rd = c["rotary_dim"] or c["head_dim"]
    theta = c["theta"]
    if c["scaling"] == "ntk":
        theta *= c["factor"] ** (rd / (rd - 2))
    w = [theta ** (-2.0 * i / rd) for i in range(rd // 2)]
    if c["scaling"] == "linear":
        w = [x / c["factor"] for x in w]
    if c["scaling"] == "by_parts":  # turns over the trained context: 1 or fewer slow down, 32 or more stay
        def part(x):
            g = min(1.0, max(0.0, (c["trained"] * x / (2 * math.pi) - 1.0) / 31.0))
            return (1 - g) * x / c["factor"] + g * x
        w = [part(x) for x in w]
    return torch.tensor(w, dtype=torch.float64, device="cuda")


def prepare(case, seed):
    c = dict(_DEFAULTS, **case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, d, hq, hk, page = _dt(c), c["head_dim"], c["q_heads"], c["kv_heads"], c["page"]
    new, held = _lengths(c)
    t, n = sum(new), c["seqs"]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": c, "t": t, "pos0": ints(held)}
    s["cu"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    s["cu"][1:] = torch.cumsum(ints(new), 0)
    s["longest"] = max(a + b for a, b in zip(new, held))
    s["most_new"] = max(new)
    s["held_rows"] = sum(new) + sum(held)
    # a fused projection's rows, a few key channels far larger than the rest
    loud = torch.ones(hk, d, device="cuda")
    loud[:, :: max(1, d // 4)] = 4.0
    rows = randn(t, hq + 2 * hk, d)
    rows[:, hq:hq + hk] *= loud
    rows = rows.to(dt)
    s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
    if c["kind"] == "rotary" or (c["kind"] == "cache" and c["rotate"]):
        angle = torch.arange(s["longest"], dtype=torch.float64, device="cuda")[:, None] * _frequencies(c)
        s["cos"] = (torch.cos(angle) * c["attention_factor"]).float()
        s["sin"] = (torch.sin(angle) * c["attention_factor"]).float()
    if c["kind"] != "rotary":
        # pages in scattered order, a few that nobody holds; what is held is quantised page by page
        cols = -(-s["longest"] // page)
        need = [-(-(a + b) // page) for a, b in zip(new, held)]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((n, cols), n_pages - 1, dtype=torch.int32, device="cuda")
        at = 0
        for b in range(n):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        s["table"] = table
        for name, gain in (("k", loud[:, None, :]), ("v", 1.0)):
            x = randn(n_pages, hk, page, d) * gain
            scale = x.abs().amax((2, 3)) * (1 / 127)
            s[name + "_scales"] = scale
            s[name + "_pages"] = torch.round(x / scale[:, :, None, None]).clamp(-127, 127).to(torch.int8)
            del x
    if c["kind"] == "cache":
        s["all_cu"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        s["all_cu"][1:] = torch.cumsum(ints([a + b for a, b in zip(new, held)]), 0)
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a serving program keeps between calls: the table of turns, its buffers, the prepared calls."""
    import paper_2606_07684_amd as scd

    c = s["case"]
    batch = scd.Batch(s["t"], s["cu"], s["pos0"])
    table = None
    if "cos" in s:
        rotary = scd.Rotary(c["head_dim"], c["theta"], rotary_dim=c["rotary_dim"] or None,
                            layout=c["layout"], scaling=c["scaling"], factor=c["factor"],
                            trained_positions=c["trained"], attention_factor=c["attention_factor"])
        table = scd.scd_rotary_table(rotary, s["longest"])
    empty = lambda rows, heads: torch.empty(rows, heads, c["head_dim"], dtype=_dt(c), device="cuda")  # noqa: E731
    if c["kind"] == "rotary":
        s["out"] = (empty(s["t"], c["q_heads"]), empty(s["t"], c["kv_heads"]))
        s["calls"] = [scd.prepare_rotary(table, batch, s["q"], s["k"], *s["out"],
                                         transpose=c["transpose"])]
        return
    cache = scd.PagedCache(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["table"])
    if c["kind"] == "cache":
        s["out"] = (empty(s["held_rows"], c["kv_heads"]), empty(s["held_rows"], c["kv_heads"]),
                    s["k_scales"], s["v_scales"])
        s["calls"] = [scd.prepare_cache_append(cache, batch, s["k"], s["v"], table),
                      scd.prepare_cache_read(cache, scd.Batch(s["held_rows"], s["all_cu"]),
                                             *s["out"][:2])]
        return
    s["out"] = empty(s["t"], c["q_heads"])
    s["calls"] = [scd.prepare_cache_attend(cache, batch, s["q"], s["out"],
                                           scale=c["head_dim"] ** -0.5)]


# ---- one pass ----------------------------------------------------------------------------------
def _rows_of(cu, t):
    """The request of every packed row."""
    return torch.bucketize(torch.arange(t, dtype=torch.int32, device="cuda"), cu[1:], right=True)


def _turn(x, cos, sin, c):
    """x [rows, heads, d] in 32 bits, turned by its rows' angles."""
    rd = 2 * cos.shape[1]
    cos, sin = cos[:, None], -sin[:, None] if c["transpose"] else sin[:, None]
    first, second = (slice(0, rd // 2), slice(rd // 2, rd)) if c["layout"] == "half" else \
        (slice(0, rd, 2), slice(1, rd, 2))
    a, b = x[..., first], x[..., second]
    y = x.clone()
    y[..., first] = a * cos - b * sin
    y[..., second] = b * cos + a * sin
    return y


def _run_rotary(s):
    c = s["case"]
    req = _rows_of(s["cu"], s["t"])
    pos = torch.arange(s["t"], device="cuda") - s["cu"][req] + s["pos0"][req]
    cos, sin = s["cos"][pos], s["sin"][pos]
    return (_turn(s["q"].float(), cos, sin, c).to(_dt(c)), _turn(s["k"].float(), cos, sin, c).to(_dt(c)))


def _append(pages, scales, x, page, slot):
    """x [rows, heads, d] stored into (page, slot); a page's scale grows to hold its largest value."""
    n_pages, heads = scales.shape
    top = x.abs().amax(2)
    grown = torch.zeros_like(scales).scatter_reduce(0, page[:, None].expand(-1, heads), top, "amax")
    grown = grown * (1 / 127)
    started = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    started[page[slot == 0]] = True
    touched = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    touched[page] = True
    old = torch.where(started[:, None], torch.zeros_like(scales), scales)
    now = torch.where(touched[:, None], torch.maximum(old, grown), scales)
    now = torch.where(now < 2.0 ** -126, torch.zeros_like(now), now)
    inv = torch.where(now > 0, torch.reciprocal(now), torch.zeros_like(now))
    again = (now > old) & touched[:, None]
    kept = torch.round(pages.float() * (old * inv)[:, :, None, None]).clamp(-127, 127).to(torch.int8)
    pages.copy_(torch.where(again[:, :, None, None], kept, pages))
    scales.copy_(now)
    pages[page, :, slot] = torch.round(x * inv[page][:, :, None]).clamp(-127, 127).to(torch.int8)


def _run_cache(s):
    c = s["case"]
    size, dt = c["page"], _dt(c)
    req = _rows_of(s["cu"], s["t"])
    pos = torch.arange(s["t"], device="cuda") - s["cu"][req] + s["pos0"][req]
    page, slot = s["table"][req, pos // size].long(), pos % size
    k, v = s["k"].float(), s["v"].float()
    if c["rotate"]:
        k = _turn(k, s["cos"][pos], s["sin"][pos], c)
    _append(s["k_pages"], s["k_scales"], k, page, slot)
    _append(s["v_pages"], s["v_scales"], v, page, slot)
    req = _rows_of(s["all_cu"], s["held_rows"])
    pos = torch.arange(s["held_rows"], device="cuda") - s["all_cu"][req]
    page, slot = s["table"][req, pos // size].long(), pos % size
    back = lambda pages, scales: (pages[page, :, slot].float() * scales[page][:, :, None]).to(dt)  # noqa: E731
    return (back(s["k_pages"], s["k_scales"]), back(s["v_pages"], s["v_scales"]), s["k_scales"],
            s["v_scales"])


def _run_attend(s):
    c = s["case"]
    n, hq, hk, d, t = c["seqs"], c["q_heads"], c["kv_heads"], c["head_dim"], s["t"]
    g, most = hq // hk, s["most_new"]
    table = s["table"].long()
    full = table.shape[1] * c["page"]
    wide = lambda pages, scales: (pages[table].float() * scales[table][..., None, None]).transpose(1, 2).reshape(n, hk, full, d)  # noqa: E731
    k, v = wide(s["k_pages"], s["k_scales"]), wide(s["v_pages"], s["v_scales"])
    req = _rows_of(s["cu"], t)
    at = torch.arange(t, device="cuda") - s["cu"][req]
    q = torch.zeros(n, most, hk, g, d, device="cuda")
    q[req, at] = s["q"].float().reshape(t, hk, g, d)
    score = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(n, hk, g * most, d), k.transpose(2, 3)) * d ** -0.5
    last = s["pos0"][:, None] + torch.arange(most, device="cuda")
    hidden = torch.arange(full, device="cuda") > last[:, :, None]
    score = score.view(n, hk, g, most, full).masked_fill_(hidden[:, None, None], float("-inf"))
    score = torch.exp_(score - score.amax(4, keepdim=True))
    total = score.sum(4, keepdim=True)
    o = torch.matmul(score.view(n, hk, g * most, full), v).view(n, hk, g, most, d) / total
    return o.permute(0, 3, 1, 2, 4)[req, at].reshape(t, hq, d).to(_dt(c))


def run(state):
    if own:
        for call in state["calls"]:
            call()
        return state["out"]
    return {"rotary": _run_rotary, "cache": _run_cache, "attend": _run_attend}[state["case"]["kind"]](state)


# ---- the definition in 64 bits -------------------------------------------------------------------
def _spans(cu):
    edges = cu.tolist()
    return list(zip(edges[:-1], edges[1:]))


def _rotated64(x, first, c):
    """Rows of one request, positions from ``first``, by complex multiplication."""
    rd = c["rotary_dim"] or c["head_dim"]
    x = x.double()
    pos = torch.arange(first, first + x.shape[0], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(pos[:, None] * _frequencies(c), c["attention_factor"]),
                       pos[:, None] * _frequencies(c) * (-1 if c["transpose"] else 1))[:, None]
    part = x[..., :rd]
    if c["layout"] == "half":
        z = torch.complex(part[..., :rd // 2].contiguous(), part[..., rd // 2:].contiguous()) * turn
        y = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(part.reshape(*part.shape[:-1], rd // 2, 2).contiguous()) * turn
        y = torch.view_as_real(z).reshape(part.shape)
    return torch.cat([y, x[..., rd:]], -1)


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    c = s["case"]
    size, hk = c["page"], c["kv_heads"]
    spans, held = _spans(s["cu"]), s["pos0"].tolist()
    if c["kind"] == "rotary":
        turned = lambda x: torch.cat([_rotated64(x[a:b], h, c) for (a, b), h in zip(spans, held)])  # noqa: E731
        return turned(s["q"]), turned(s["k"])
    if c["kind"] == "attend":
        out = torch.zeros(s["t"], c["q_heads"], c["head_dim"], dtype=torch.float64, device="cuda")
        g = c["q_heads"] // hk
        for r, ((a, b), h) in enumerate(zip(spans, held)):
            if a == b:
                continue
            ids = s["table"][r, :-(-(h + b - a) // size)].long()
            late = torch.arange(h + b - a, device="cuda") > torch.arange(h, h + b - a, device="cuda")[:, None]
            for j in range(hk):
                rows = lambda n: (s[n + "_pages"][ids, j].double() * s[n + "_scales"][ids, j].double()[:, None, None]).flatten(0, 1)[:h + b - a]  # noqa: E731,B023
                k, v = rows("k"), rows("v")
                for i in range(j * g, j * g + g):
                    logit = (s["q"][a:b, i].double() @ k.T) * c["head_dim"] ** -0.5
                    out[a:b, i] = torch.softmax(logit.masked_fill(late, -math.inf), 1) @ v
        return out
    results = []
    for name in ("k", "v"):
        pages = s[name + "_pages"].double()
        scales = s[name + "_scales"].double()
        dense = []
        for r, ((a, b), h) in enumerate(zip(spans, held)):
            x = s[name][a:b].double()
            if name == "k" and c["rotate"]:
                x = _rotated64(s[name][a:b], h, c)
            for col in range(h // size, -(-(h + b - a) // size)):
                p = int(s["table"][r, col])
                lo, hi = max(h, col * size), min(h + b - a, (col + 1) * size)
                if lo >= hi:
                    continue
                rows = x[lo - h:hi - h].transpose(0, 1)
                old = scales[p] if lo > col * size else torch.zeros_like(scales[p])
                now = torch.maximum(old, rows.abs().amax((1, 2)) / 127)
                inv = torch.where(now > 0, 1 / now, torch.zeros_like(now))
                if lo > col * size:
                    ratio = torch.where(now > old, old * inv, torch.ones_like(now))
                    pages[p] = torch.round(pages[p] * ratio[:, None, None])
                pages[p, :, lo - col * size:hi - col * size] = torch.round(rows * inv[:, None, None]).clamp(-127, 127)
                scales[p] = now
            ids = s["table"][r, :-(-(h + b - a) // size)].long()
            dense.append((pages[ids] * scales[ids][:, :, None, None]).transpose(1, 2).flatten(0, 1)[:h + b - a])
        results.append((torch.cat(dense), scales))
    (k, ks), (v, vs) = results
    return k, v, ks, vs
