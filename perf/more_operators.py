"""Serving from a latent cache, and the pages of caches, as cases that a timing or comparison program can run.

A model whose layers keep one latent vector a token (and one rotated key that all heads share) caches
that row instead of keys and values.  Kinds of pass:
  append    latent rows and shared keys of new tokens, keys rotated on the way, into pages
  absorbed  new tokens' attention over the paged latents: the heads' key and value matrices are applied
            to queries and results, never to the cache
  expand    the dense keys and values of everything that requests hold, for prompts
  rows      causal attention over dense keys and values, which expansion (or the codec) has written
  fork      a step of a search: candidates are dropped, others forked in their place, every request gets
            a page for its next token, pages that it would share are copied, in every layer
  compact   the pages in use move to the front of the pool, in every layer

``run`` with ``own`` false computes the same in elementary torch operations in 32 bits; with ``own``
true it calls the framework's entry points.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(dtype="bf16", heads=32, kv_heads=32, plain=128, value=128, latent=256, turned=64, page=64,
                 theta=5e5, seqs=1, new=1, ragged=False, held_lo=0, held_hi=0, split=1,
                 layers=1, cache="latent", forks=0, spare=0, pages=0, kept=0.5)


def _case(name, kind, **kw):
    c = dict(_DEFAULTS, kind=kind)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One generated token of each of 64 requests: the smallest call, launch latency decides.
        _case("append_token", "append", seqs=64, new=64, held_lo=1, held_hi=8000),
        # Five ragged prompts in fp32, the smallest model's heads, pages of 16 tokens.
        _case("append_ragged_f32", "append", dtype="f32", latent=64, turned=32, page=16, theta=1e4, seqs=5,
              new=10007, ragged=True),
        # One token of one short request: latency decides.
        _case("absorbed_token_short", "absorbed", held_lo=332, held_hi=332),
        # One token of each of 16 requests with 1K to 16K tokens: the bulk of generation.
        _case("absorbed_token_batch", "absorbed", seqs=16, new=16, held_lo=1023, held_hi=16383),
        # A few proposed tokens of each of 8 requests, fp32, few heads, small pages.
        _case("absorbed_few_f32", "absorbed", dtype="f32", heads=8, plain=64, value=64, latent=64, turned=32,
              page=16, theta=1e4, seqs=8, new=37, ragged=True, held_lo=50, held_hi=1500),
        # Five prefixes, 20000 tokens in all, of 28 heads and a rank of 96.
        _case("expand_prefixes", "expand", heads=28, latent=96, theta=1e6, seqs=5, new=20000, ragged=True),
        # One 1000-token prefix in fp32 of the smallest heads.
        _case("expand_f32", "expand", dtype="f32", heads=8, plain=64, value=64, latent=64, turned=32, page=16,
              theta=1e4, new=1000),
        # The last 2048 tokens of an 8192-token prompt, keys of 128 + 64 channels, values of 128.
        _case("rows_prompt", "rows", new=2048, held_lo=6144, held_hi=6144),
        # Ragged prompts of the codec's own rows: 8 key heads of 128 for 32, no expansion.
        _case("rows_ragged", "rows", kv_heads=8, turned=0, seqs=3, new=2500, ragged=True, held_hi=1500),
        # Four candidates of one request, two layers of the 8-bit cache: latency decides.
        _case("fork_few", "fork", cache="bytes", kv_heads=4, plain=64, page=16, layers=2, seqs=1, forks=3,
              held_lo=332, held_hi=332, spare=8),
        # 16 requests of four candidates each, 32 layers of latents.
        _case("fork_batch", "fork", layers=32, seqs=16, forks=3, held_lo=100, held_hi=1500, spare=100),
        # Half of the pool's pages are free and scattered, 16 layers of the 8-bit cache.
        _case("compact_half", "compact", cache="bytes", kv_heads=8, layers=16, seqs=24, pages=512, kept=0.5),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "absorbed", "absorbed", "absorbed", "expand", "rows", "rows", "fork", "compact"])
    heads, plain, value, latent, turned, theta = rng.choice(
        [(32, 128, 128, 256, 64, 5e5), (28, 128, 128, 96, 64, 1e6), (64, 128, 128, 128, 64, 5e5),
         (8, 64, 64, 64, 32, 1e4), (16, 64, 128, 256, 32, 1e4)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = _case(None, kind, dtype=dtype, heads=heads, kv_heads=heads, plain=plain, value=value, latent=latent,
              turned=turned, theta=theta, page=rng.choice([16, 32, 64, 128]), split=rng.randrange(1 << 20))
    if kind == "append":
        new = _between(rng, 1, 30000)
        c.update(seqs=min(new, _between(rng, 1, 64)), new=new, ragged=rng.random() < 0.7, held_hi=rng.randrange(300))
    elif kind == "absorbed" and rng.random() < 0.75:  # a token, or a few, of each request
        seqs = _between(rng, 1, 64)
        held = _between(rng, 32, min(32000, 130000 // seqs))
        c.update(seqs=seqs, new=seqs * rng.choice([1, 1, 1, 2, 5]), ragged=rng.random() < 0.5,
                 held_lo=held // 8, held_hi=held)
    elif kind == "absorbed":  # a chunk behind what is held
        c.update(seqs=rng.choice([1, 2]), new=_between(rng, 16, 200), ragged=rng.random() < 0.7,
                 held_hi=rng.randrange(3000))
    elif kind == "expand":
        new = _between(rng, 1, 16000) if dtype == "bf16" else _between(rng, 1, 1500)
        c.update(seqs=min(new, _between(rng, 1, 16)), new=new, ragged=rng.random() < 0.7)
    elif kind == "rows":
        if rng.random() < 0.4:  # the codec's rows, grouped heads
            heads, group = rng.choice([(32, 4), (28, 7), (8, 2)])
            plain = rng.choice([64, 128])
            c.update(heads=heads, kv_heads=heads // group, plain=plain, value=plain, turned=0)
        if rng.random() < 0.3:
            seqs = _between(rng, 1, 16)
            c.update(seqs=seqs, new=seqs, held_hi=_between(rng, 32, 16000 // seqs))
        else:
            most = 1500 if dtype == "bf16" else 500
            c.update(seqs=rng.choice([1, 1, 2, 3]), new=_between(rng, 16, most), ragged=rng.random() < 0.7,
                     held_hi=rng.randrange(2 * most))
    elif kind == "fork":
        seqs = _between(rng, 1, 24)
        c.update(dtype="bf16", cache=rng.choice(["latent", "bytes"]), kv_heads=rng.choice([4, 8]),
                 layers=_between(rng, 1, 24), seqs=seqs, forks=rng.randrange(1, 5), held_lo=rng.randrange(1, 200),
                 held_hi=rng.randrange(200, 1200), spare=rng.randrange(40, 120))
        if c["cache"] == "bytes":
            c.update(page=rng.choice([16, 32, 64]))
    else:
        c.update(dtype="bf16", cache=rng.choice(["latent", "bytes"]), kv_heads=rng.choice([4, 8]),
                 layers=_between(rng, 1, 16), seqs=_between(rng, 1, 64), pages=_between(rng, 8, 500),
                 kept=rng.uniform(0.1, 0.95))
        if c["cache"] == "bytes":
            c.update(page=rng.choice([16, 32, 64]))
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


def _page_bytes(c):
    """Bytes of a page in all layers."""
    if c["cache"] == "bytes":
        return c["layers"] * 2 * c["kv_heads"] * (c["page"] * c["plain"] + 4)
    return c["layers"] * c["page"] * (c["latent"] + c["turned"]) * (2 if c["dtype"] == "bf16" else 4)


def _used(c):
    """Pages in use of a pool that is to be compacted."""
    return max(1, int(c["pages"] * c["kept"]))


def work(case):
    c = dict(_DEFAULTS, **case)
    new, held = _lengths(c)
    eb = 2 if c["dtype"] == "bf16" else 4
    h, dn, dv, r, dr, t = c["heads"], c["plain"], c["value"], c["latent"], c["turned"], sum(new)
    kv = sum(n + m for n, m in zip(new, held))
    pairs = sum(n * m + n * (n + 1) // 2 for n, m in zip(new, held))
    weights = h * (dn + dv) * r * eb
    if c["kind"] == "append":
        return {"bytes": 2 * t * (r + dr) * eb, "flops": 3 * t * dr}
    if c["kind"] == "absorbed":
        return {"bytes": kv * (r + dr) * eb + weights + t * h * (dn + dr + dv) * eb,
                "flops": 2.0 * h * (pairs * (2 * r + dr) + t * r * (dn + dv))}
    if c["kind"] == "expand":
        return {"bytes": t * (r + dr) * eb + weights + t * h * (dn + dr + dv) * eb,
                "flops": 2.0 * t * h * r * (dn + dv)}
    if c["kind"] == "rows":
        return {"bytes": (kv * c["kv_heads"] + t * h) * (dn + dr + dv) * eb,
                "flops": 2.0 * h * pairs * (dn + dr + dv)}
    if c["kind"] == "fork":
        # every fork whose last page is begun ends in one page copied; tables are read and written
        moves = sum(c["forks"] for n in held if n % c["page"])
        rows = sum((1 + 3 * c["forks"]) * (-(-(n + 1) // c["page"])) for n in held)
        return {"bytes": 2 * moves * _page_bytes(c) + 8 * rows, "flops": rows}
    order = random.Random(c["split"]).sample(range(c["pages"]), _used(c))
    moves = sum(p >= len(order) for p in order)
    return {"bytes": 2 * moves * _page_bytes(c) + 16 * c["pages"], "flops": c["pages"]}


# ---- inputs ------------------------------------------------------------------------------------
def _angles(c, most):
    w = [c["theta"] ** (-2.0 * i / c["turned"]) for i in range(c["turned"] // 2)]
    return torch.arange(most, dtype=torch.float64, device="cuda")[:, None] * \
        torch.tensor(w, dtype=torch.float64, device="cuda")


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _edges(lengths):
    cu = torch.zeros(len(lengths) + 1, dtype=torch.int32, device="cuda")
    cu[1:] = torch.cumsum(_ints(lengths), 0)
    return cu


def prepare(case, seed):
    c = dict(_DEFAULTS, **case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["kind"] in ("fork", "compact"):
        _prepare_pages(s, gen, seed)
    else:
        dt, h, dn, dv, r, dr = _dt(c), c["heads"], c["plain"], c["value"], c["latent"], c["turned"]
        new, held = _lengths(c)
        t, n, page = sum(new), c["seqs"], c["page"]
        s.update(t=t, cu=_edges(new), pos0=_ints(held), most_new=max(new), rows=sum(new) + sum(held),
                 longest=max(a + b for a, b in zip(new, held)))
        if c["kind"] == "append":  # a fused projection's rows: the latent, then the shared key
            rows = randn(t, r + dr).to(dt)
            s["c"], s["k"] = rows[:, :r], rows[:, r:]
            angle = _angles(c, s["longest"])
            s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
        if c["kind"] in ("absorbed", "rows"):
            s["q"] = randn(t, h, dn + dr).to(dt)
        if c["kind"] in ("absorbed", "expand"):
            s["w_k"], s["w_v"] = ((randn(h, d, r) * r ** -0.5).to(dt) for d in (dn, dv))
        if c["kind"] == "rows":
            s["all_cu"] = _edges([a + b for a, b in zip(new, held)])
            s["k"], s["v"] = (randn(s["rows"], c["kv_heads"], d).to(dt) for d in (dn + dr, dv))
        else:  # pages in scattered order, a few that nobody holds
            need = [-(-(a + b) // page) for a, b in zip(new, held)]
            n_pages, cols = sum(need) + 3, -(-s["longest"] // page)
            order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
            table = torch.full((n, cols), n_pages - 1, dtype=torch.int32, device="cuda")
            at = 0
            for b in range(n):
                table[b, :need[b]] = order[at:at + need[b]]
                at += need[b]
            s["table"] = table
            s["pages"] = randn(n_pages, page, r + dr).to(dt)
    if own:
        _plan(s)
    return s


def _prepare_pages(s, gen, seed):
    """Tables, counts of references, held tokens, and the pages of every layer."""
    c = s["case"]
    page, rng = c["page"], random.Random(c["split"] if c["kind"] == "compact" else seed)
    if c["kind"] == "fork":
        # request i holds its tokens; its candidates, the rows behind all requests, were forked before
        # and hold its pages but the last, of which each has a copy
        _, held = _lengths(c)
        owners = held + [n for n in held for _ in range(c["forks"])]
        full = [n // page for n in owners]
        cols = max(-(-(n + 1) // page) for n in owners)
        n_pages = sum(full[:c["seqs"]]) + len(owners) + c["spare"]
        order = random.Random(seed).sample(range(n_pages), n_pages)
        table = []
        for i, n in enumerate(owners):
            shared = table[(i - c["seqs"]) // c["forks"]][:full[i]] if i >= c["seqs"] else \
                [order.pop() for _ in range(full[i])]
            table.append(shared + [order.pop()] + [-1] * (cols - full[i] - 1))
        s["src"] = _ints([i for i in range(c["seqs"]) for _ in range(c["forks"])])
        s["dst"] = _ints(list(range(c["seqs"], len(owners))))
        s["cu"] = torch.arange(len(owners) + 1, dtype=torch.int32, device="cuda")
    else:
        # requests of any lengths hold the pool's used pages in scattered order
        n_pages, used = c["pages"], _used(c)
        order = rng.sample(range(n_pages), used)
        cuts = sorted(rng.randrange(used + 1) for _ in range(c["seqs"] - 1))
        runs = [order[a:b] for a, b in zip([0] + cuts, cuts + [used])]
        cols = max(len(x) for x in runs)
        owners = [len(x) * page for x in runs]
        table = [x + [-1] * (cols - len(x)) for x in runs]
    refs = [0] * n_pages
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    s["table"], s["refs"], s["held"] = _ints(table), _ints(refs), _ints(owners)
    s["table0"], s["refs0"] = s["table"].clone(), s["refs"].clone()
    most = max(len(owners), n_pages // 2 + 1)
    s["moves"] = torch.zeros(most, 2, dtype=torch.int32, device="cuda")
    s["status"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    # every layer's pages one behind another
    if c["cache"] == "bytes":
        shape = (c["layers"], n_pages, c["kv_heads"], page, c["plain"])
        s["planes"] = (*(torch.randint(-127, 128, shape, generator=gen, dtype=torch.int8, device="cuda") for _ in "kv"),
                       *(torch.rand(shape[:3], generator=gen, device="cuda") for _ in "kv"))
    else:
        shape = (c["layers"], n_pages, page, c["latent"] + c["turned"])
        s["planes"] = (torch.randn(shape, generator=gen, device="cuda").to(_dt(c)),)


def _plan(s):
    """What a serving program keeps between calls: tables of turns, its buffers, the prepared calls."""
    import paper_2606_07684_amd as scd

    c = s["case"]
    if c["kind"] in ("fork", "compact"):
        pages = scd.Pages(s["table"], s["refs"], s["held"], c["page"])
        moves = scd.Moves(s["moves"], s["status"])
        caches = [scd.PagedCache(*x, s["table"]) if c["cache"] == "bytes" else
                  scd.LatentCache(x[0], s["table"], c["latent"]) for x in zip(*s["planes"])]
        copy = scd.prepare_pages_copy(caches, moves)
        if c["kind"] == "compact":
            before = scd.Pages(s["table0"], s["refs0"], s["held"], c["page"])
            s["calls"] = [scd.prepare_pages_compact(before, moves, out=pages), copy]
        else:
            one = scd.Batch(s["held"].numel(), s["cu"], s["held"])
            s["calls"] = [scd.prepare_pages_free(pages, s["dst"]), scd.prepare_pages_fork(pages, s["src"], s["dst"]),
                          scd.prepare_pages_reserve(pages, one, moves), copy]
        return
    batch = scd.Batch(s["t"], s["cu"], s["pos0"])
    empty = lambda *shape: torch.empty(shape, dtype=_dt(c), device="cuda")  # noqa: E731
    h, dn, dv, dr = c["heads"], c["plain"], c["value"], c["turned"]
    if c["kind"] == "rows":
        s["out"] = empty(s["t"], h, dv)
        s["calls"] = [scd.prepare_rows_attend(batch, scd.Batch(s["rows"], s["all_cu"]), s["q"], s["k"], s["v"],
                                              s["out"], scale=(dn + dr) ** -0.5)]
        return
    cache = scd.LatentCache(s["pages"], s["table"], c["latent"])
    if c["kind"] == "append":
        table = scd.scd_rotary_table(scd.Rotary(dr, c["theta"]), s["longest"])
        s["calls"] = [scd.prepare_latent_append(cache, batch, s["c"], s["k"], table)]
        s["out"] = s["pages"]
    elif c["kind"] == "expand":
        s["out"] = empty(s["t"], h, dn + dr), empty(s["t"], h, dv)
        s["calls"] = [scd.prepare_latent_expand(cache, batch, s["w_k"], s["w_v"], *s["out"])]
    else:
        s["out"] = empty(s["t"], h, dv)
        s["calls"] = [scd.prepare_latent_attend(cache, batch, s["q"], s["w_k"], s["w_v"], s["out"],
                                                scale=(dn + dr) ** -0.5)]


# ---- one pass ----------------------------------------------------------------------------------
def _rows_of(cu, t):
    """The request of every packed row."""
    return torch.bucketize(torch.arange(t, dtype=torch.int32, device="cuda"), cu[1:], right=True)


def _places(s):
    """Request, page and slot of every row of the batch."""
    size = s["case"]["page"]
    req = _rows_of(s["cu"], s["t"])
    pos = torch.arange(s["t"], device="cuda") - s["cu"][req] + s["pos0"][req]
    return pos, s["table"][req, pos // size].long(), pos % size


def _run_append(s):
    dt = s["pages"].dtype
    pos, page, slot = _places(s)
    cos, sin = s["cos"][pos], s["sin"][pos]
    a, b = s["k"].float().chunk(2, 1)
    s["pages"][page, slot] = torch.cat([s["c"], (a * cos - b * sin).to(dt), (b * cos + a * sin).to(dt)], 1)
    return s["pages"]


def _softmax_rows(score, limit):
    """Weights of scores [n, ..., most, full], of the positions up to limit [n, most]."""
    n, most, full = score.shape[0], score.shape[-2], score.shape[-1]
    hidden = (torch.arange(full, device="cuda") > limit[:, :, None]).view(n, *([1] * (score.dim() - 3)), most, full)
    score = score.masked_fill_(hidden, float("-inf"))
    score = torch.exp_(score - score.amax(-1, keepdim=True))
    return score.div_(score.sum(-1, keepdim=True))


def _run_absorbed(s):
    c = s["case"]
    n, h, dn, r, t, most = c["seqs"], c["heads"], c["plain"], c["latent"], s["t"], s["most_new"]
    held = s["pages"][s["table"].long()].float().flatten(1, 2)  # [n, full, r + turned]
    req = _rows_of(s["cu"], t)
    at = torch.arange(t, device="cuda") - s["cu"][req]
    q = s["q"].float()
    q = torch.cat([torch.matmul(q[..., :dn].transpose(0, 1), s["w_k"].float()).transpose(0, 1), q[..., dn:]], -1)
    wide = torch.zeros(n, h, most, q.shape[2], device="cuda")
    wide[req, :, at] = q
    score = torch.matmul(wide.flatten(1, 2), held.transpose(1, 2)) * (dn + c["turned"]) ** -0.5
    weights = _softmax_rows(score.view(n, h, most, -1), s["pos0"][:, None] + torch.arange(most, device="cuda"))
    o = torch.matmul(weights.flatten(1, 2), held[..., :r]).view(n, h, most, r)[req, :, at]
    o = torch.matmul(o.transpose(0, 1), s["w_v"].float().transpose(1, 2))
    return o.transpose(0, 1).to(_dt(c)).contiguous()


def _run_expand(s):
    c = s["case"]
    _, page, slot = _places(s)
    rows = s["pages"][page, slot]
    x, h, r = rows[:, :c["latent"]].float(), c["heads"], c["latent"]
    k = torch.matmul(x, s["w_k"].float().view(-1, r).t()).view(-1, h, c["plain"]).to(_dt(c))
    v = torch.matmul(x, s["w_v"].float().view(-1, r).t()).view(-1, h, c["value"]).to(_dt(c))
    return torch.cat([k, rows[:, None, r:].expand(-1, h, -1)], 2), v


def _run_rows(s):
    c = s["case"]
    n, h, hk, t, most, full = c["seqs"], c["heads"], c["kv_heads"], s["t"], s["most_new"], s["longest"]
    req, owner = _rows_of(s["cu"], t), _rows_of(s["all_cu"], s["rows"])
    at = torch.arange(t, device="cuda") - s["cu"][req]
    place = torch.arange(s["rows"], device="cuda") - s["all_cu"][owner]
    def wide(x, r, i, m):  # [n, heads, m, channels]
        y = torch.zeros(n, x.shape[1], m, x.shape[2], device="cuda")
        y[r, :, i] = x.float()
        return y
    q, k, v = wide(s["q"], req, at, most), wide(s["k"], owner, place, full), wide(s["v"], owner, place, full)
    score = torch.matmul(q.view(n, hk, -1, q.shape[3]), k.transpose(2, 3)) * q.shape[3] ** -0.5
    weights = _softmax_rows(score.view(n, h, most, full), s["pos0"][:, None] + torch.arange(most, device="cuda"))
    o = torch.matmul(weights.view(n, hk, -1, full), v).view(n, h, most, -1)
    return o[req, :, at].to(_dt(c))


def _copy_pages(s):
    pairs = s["moves"][:int(s["status"][0])].long()
    for plane in s["planes"]:
        plane[:, pairs[:, 1]] = plane[:, pairs[:, 0]]


def _count(refs, ids, by):
    refs.scatter_add_(0, ids.clamp(min=0).flatten().long(), torch.where(ids >= 0, by, 0).flatten().to(torch.int32))


def _run_fork(s):
    table, refs, held, size = s["table"], s["refs"], s["held"], s["case"]["page"]
    src, dst = s["src"].long(), s["dst"].long()
    # the candidates give their pages back, and take those that their sources' tokens are in
    _count(refs, table[dst], -1)
    columns = torch.arange(table.shape[1], device="cuda")
    taken = torch.where(columns * size < held[src][:, None], table[src], -1)
    table[dst], held[dst] = taken, held[src]
    _count(refs, taken, 1)
    # pages that the next tokens go to: missing ones, and in place of shared ones
    new = s["cu"][1:] - s["cu"][:-1]
    want = (columns >= (held // size)[:, None]) & (columns * size < (held + new)[:, None])
    ids = torch.where(want & (table >= 0), table, refs.numel()).flatten()
    order = torch.sort(ids, stable=True)
    place = torch.arange(ids.numel(), device="cuda")
    rank = torch.empty_like(place)
    rank[order.indices] = place - torch.searchsorted(order.values, order.values)
    named = (ids < refs.numel()).view_as(table)
    shared = named & (refs[table.clamp(min=0)] - rank.view_as(table) > 1)
    take = (want & (table < 0)) | shared
    free = torch.sort((refs > 0).int(), stable=True).indices.to(torch.int32)
    fresh = torch.where(take, free[(torch.cumsum(take.flatten(), 0) - 1).clamp(min=0)].view_as(table), table)
    copied = shared & (columns * size < held[:, None])
    pairs = torch.stack([table[copied], fresh[copied]], 1)
    s["moves"][:pairs.shape[0]] = pairs
    s["status"].copy_(torch.stack([copied.sum(), *[torch.zeros_like(rank[0])] * 3]))
    _count(refs, torch.where(shared, table, -1), -1)
    _count(refs, torch.where(take, fresh, -1), 1)
    table.copy_(fresh)
    _copy_pages(s)


def _run_compact(s):
    table, refs, moves = s["table0"], s["refs0"], s["moves"]
    used = refs > 0
    n = used.sum()
    place = torch.arange(refs.numel(), device="cuda")
    high, hole = (used & (place >= n)).nonzero()[:, 0], (~used & (place < n)).nonzero()[:, 0]
    to = place.clone()
    to[high] = hole
    moves[:high.numel()] = torch.stack([high, hole], 1).to(torch.int32)
    s["status"].copy_(torch.stack([torch.full_like(n, high.numel()), n, *[torch.zeros_like(n)] * 2]))
    s["table"].copy_(torch.where(table >= 0, to[table.clamp(min=0)], -1))
    counts = torch.where(place < n, refs, 0)
    counts[hole] = refs[high]
    s["refs"].copy_(counts)
    _copy_pages(s)


def run(state):
    kind = state["case"]["kind"]
    if own:
        for call in state["calls"]:
            call()
        if "out" in state:
            return state["out"]
    elif kind not in ("fork", "compact"):
        return {"append": _run_append, "absorbed": _run_absorbed, "expand": _run_expand, "rows": _run_rows}[kind](state)
    else:
        (_run_fork if kind == "fork" else _run_compact)(state)
    return {k: state[k] for k in ("table", "refs", "held", "moves", "status", "planes")}


# ---- the definition in 64 bits -------------------------------------------------------------------
def _spans(cu):
    edges = cu.tolist()
    return list(zip(edges[:-1], edges[1:]))


def _held_rows(s, r, upto):
    """The first ``upto`` rows that request r holds, in 64 bits."""
    ids = s["table"][r, :-(-upto // s["case"]["page"])].long()
    return s["pages"][ids].flatten(0, 1)[:upto].double()


def _attend64(q, k, v, held, scale):
    """Rows q [n, d] behind ``held`` positions over k, v."""
    late = torch.arange(k.shape[0], device="cuda") > torch.arange(held, held + q.shape[0], device="cuda")[:, None]
    return torch.softmax((q @ k.T * scale).masked_fill(late, -math.inf), 1) @ v


def _exact_pages(s):
    """The bookkeeping one request and one page after another."""
    c = s["case"]
    size = c["page"]
    moves = s["moves"].tolist()
    status = [0, 0, 0, 0]
    if c["kind"] == "fork":
        table, refs, held = s["table"].tolist(), s["refs"].tolist(), s["held"].tolist()
        for d in s["dst"].tolist():
            for p in table[d]:
                if p >= 0:
                    refs[p] -= 1
            table[d] = [-1] * len(table[d])
        for a, d in zip(s["src"].tolist(), s["dst"].tolist()):
            held[d] = held[a]
            for j in range(-(-held[a] // size)):
                table[d][j] = table[a][j]
                refs[table[d][j]] += 1
        free = [p for p, n in enumerate(refs) if n == 0][::-1]
        for b, row in enumerate(table):
            for j in range(held[b] // size, held[b] // size + 1):
                p = row[j]
                if p >= 0 and refs[p] == 1:
                    continue
                row[j] = free.pop()
                refs[row[j]] = 1
                if p >= 0:
                    refs[p] -= 1
                    if j * size < held[b]:
                        moves[status[0]] = [p, row[j]]
                        status[0] += 1
    else:
        table, refs, held = s["table0"].tolist(), s["refs0"].tolist(), s["held"].tolist()
        n = sum(x > 0 for x in refs)
        status[1] = n
        holes = [p for p in range(n) if refs[p] == 0][::-1]
        to = {-1: -1}
        for p in range(len(refs)):
            to[p] = p
            if p >= n and refs[p] > 0:
                to[p] = holes.pop()
                moves[status[0]] = [p, to[p]]
                status[0] += 1
                refs[to[p]], refs[p] = refs[p], 0
        table = [[to[p] for p in row] for row in table]
    for a, b in moves[:status[0]]:
        for plane in s["planes"]:
            plane[:, b] = plane[:, a]
    return {"table": _ints(table), "refs": _ints(refs), "held": _ints(held), "moves": _ints(moves),
            "status": _ints(status),
            "planes": tuple(p.double() if p.is_floating_point() else p for p in s["planes"])}


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    c = s["case"]
    if c["kind"] in ("fork", "compact"):
        return _exact_pages(s)
    spans, held = _spans(s["cu"]), s["pos0"].tolist()
    h, dn, dv, r, dr, size = c["heads"], c["plain"], c["value"], c["latent"], c["turned"], c["page"]
    if c["kind"] == "append":
        pages = s["pages"].double()
        for b, ((first, last), n) in enumerate(zip(spans, held)):
            if first == last:
                continue
            angle = _angles(c, n + last - first)[n:]
            k = s["k"][first:last].double()
            turned = torch.complex(k[:, :dr // 2].contiguous(), k[:, dr // 2:].contiguous()) * \
                torch.polar(torch.ones_like(angle), angle)
            row = torch.cat([s["c"][first:last].double(), turned.real, turned.imag], 1)
            pos = torch.arange(n, n + last - first, device="cuda")
            pages[s["table"][b, pos // size].long(), pos % size] = row
        return pages
    if c["kind"] == "expand":
        k = torch.empty(s["t"], h, dn + dr, dtype=torch.float64, device="cuda")
        v = torch.empty(s["t"], h, dv, dtype=torch.float64, device="cuda")
        for b, (first, last) in enumerate(spans):
            if first == last:
                continue
            x = _held_rows(s, b, last - first)
            for i in range(h):
                k[first:last, i, :dn] = x[:, :r] @ s["w_k"][i].double().T
                k[first:last, i, dn:] = x[:, r:]
                v[first:last, i] = x[:, :r] @ s["w_v"][i].double().T
        return k, v
    out = torch.zeros(s["t"], h, dv, dtype=torch.float64, device="cuda")
    for b, ((first, last), n) in enumerate(zip(spans, held)):
        if first == last:
            continue
        if c["kind"] == "absorbed":  # by way of each head's own keys and values
            x = _held_rows(s, b, n + last - first)
        else:
            lo, hi = _spans(s["all_cu"])[b]
        for i in range(h):
            if c["kind"] == "absorbed":
                k = torch.cat([x[:, :r] @ s["w_k"][i].double().T, x[:, r:]], 1)
                v = x[:, :r] @ s["w_v"][i].double().T
            else:
                j = i // (h // c["kv_heads"])
                k, v = s["k"][lo:hi, j].double(), s["v"][lo:hi, j].double()
            out[first:last, i] = _attend64(s["q"][first:last, i].double(), k, v, n, (dn + dr) ** -0.5)
    return out
