"""A consumer that serves from what it received: decoded prefixes become a paged 8-bit cache, a prompt
is read behind them, and tokens are generated one by one from a captured step.

    python examples/serve_prefix.py

Codes and weights are random (no trained pair is available), so the numbers mean nothing; the calls
and their order are a serving program's:

1. ``scd_reuse_decode`` rebuilds every layer's keys (rotated) and values from the codes,
2. ``scd_cache_append`` puts them into pages, as they are,
3. for the prompt, layer by layer: queries, keys and values of the new tokens by the consumer's
   weights, ``scd_rotary`` on the queries, ``scd_cache_append`` with the keys rotated on the way,
   ``scd_cache_attend`` over prefix and prompt,
4. the same three calls for one token of every request, captured once as a HIP graph and replayed
   while the positions grow in device memory,
5. ``scd_cache_read`` gives the keys and values back as the dense rows that ``scd_encode`` takes,
   should this model be the producer of the next hop.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_07684_amd as scd  # noqa: E402

LAYERS, D_MODEL, HEADS, KV_HEADS, HEAD_DIM, PAGE, THETA = 4, 512, 8, 4, 64, 16, 1e4
PREFIX, PROMPT, STEPS = (300, 77, 130), (20, 1, 45), 12


def serve(seed: int = 0):
    """Runs all of the above; returns what a test looks at."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    starts = lambda lens: ints([sum(lens[:i]) for i in range(len(lens) + 1)])  # noqa: E731
    n, width, rank, longest = len(PREFIX), KV_HEADS * HEAD_DIM, 32, max(PREFIX) + max(PROMPT) + STEPS

    # 1. the prefixes' keys and values from their codes
    model = scd.Model(LAYERS, D_MODEL, KV_HEADS, HEAD_DIM, THETA, "bf16", [0] * LAYERS, [rank] * LAYERS,
                      [rank] * LAYERS, [rank] * LAYERS)
    prefix = scd.Batch(sum(PREFIX), starts(PREFIX))
    each = lambda *shape: [randn(*shape).bfloat16() for _ in range(LAYERS)]  # noqa: E731
    dense = [[torch.empty(sum(PREFIX), width, dtype=torch.bfloat16, device=dev) for _ in range(LAYERS)]
             for _ in "kv"]
    bases = [[w * rank ** -0.5 for w in each(width, rank)] for _ in "kv"]
    scd.scd_reuse_decode(model, prefix, scd.scd_rope_table(model, longest), each(sum(PREFIX), rank),
                         each(sum(PREFIX), rank), *bases, None, None, *dense)

    # 2. into pages (of every layer the same ones)
    columns = -(-longest // PAGE)
    table = torch.randperm(n * columns, generator=gen, device=dev).to(torch.int32).view(n, columns)
    caches = []
    for k, v in zip(*dense):
        pages = [torch.empty(n * columns, KV_HEADS, PAGE, HEAD_DIM, dtype=torch.int8, device=dev) for _ in "kv"]
        scales = [torch.zeros(n * columns, KV_HEADS, device=dev) for _ in "kv"]
        caches.append(scd.PagedCache(*pages, *scales, table))
        rows = [x.view(-1, KV_HEADS, HEAD_DIM) for x in (k, v)]
        scd.scd_cache_append(caches[-1], prefix, *rows)

    # 3. and 4.: the layers of a step over a batch of new tokens, its calls prepared once
    turns = scd.scd_rotary_table(scd.Rotary(HEAD_DIM, THETA), longest)
    w_qkv = [w * D_MODEL ** -0.5 for w in each((HEADS + 2 * KV_HEADS) * HEAD_DIM, D_MODEL)]
    w_out = [w * (HEADS * HEAD_DIM) ** -0.5 for w in each(D_MODEL, HEADS * HEAD_DIM)]

    def step(batch, hidden):
        """A function that runs every layer on ``hidden`` [n_tokens, D_MODEL], in place."""
        t = batch.n_tokens
        qkv = torch.empty(t, HEADS + 2 * KV_HEADS, HEAD_DIM, dtype=torch.bfloat16, device=dev)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
        attended = torch.empty(t, HEADS, HEAD_DIM, dtype=torch.bfloat16, device=dev)
        rotate = scd.prepare_rotary(turns, batch, q, None, q, None)
        appends = [scd.prepare_cache_append(c, batch, k, v, turns) for c in caches]
        workspace = torch.zeros(max(16, scd.scd_cache_attend_workspace_bytes(caches[0], batch, HEADS)),
                                dtype=torch.uint8, device=dev)
        attends = [scd.prepare_cache_attend(c, batch, q, attended, workspace=workspace) for c in caches]

        def run():
            for l in range(LAYERS):
                torch.mm(hidden, w_qkv[l].t(), out=qkv.view(t, -1))
                rotate()
                appends[l]()
                attends[l]()
                hidden.add_(torch.mm(attended.view(t, -1), w_out[l].t()))
                hidden.mul_(torch.rsqrt(hidden.float().square().mean(1, keepdim=True)).bfloat16())
        return run

    prompt = randn(sum(PROMPT), D_MODEL).bfloat16()
    first = prompt.clone()
    step(scd.Batch(sum(PROMPT), starts(PROMPT), ints(PREFIX)), prompt)()

    token = prompt[starts(PROMPT)[1:].long() - 1].contiguous()
    pos0 = ints([a + b for a, b in zip(PREFIX, PROMPT)])
    generate = step(scd.Batch(n, ints(list(range(n + 1))), pos0), token)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    kept = token.clone()
    with torch.cuda.graph(graph):
        generate()
        pos0.add_(1)
    token.copy_(kept)  # capturing runs nothing, but keep the example's state in one place
    tokens = []
    for _ in range(STEPS):
        graph.replay()
        tokens.append(token.clone())

    # 5. everything the first layer holds, as dense rows
    held = [a + b + STEPS for a, b in zip(PREFIX, PROMPT)]
    back = [torch.empty(sum(held), KV_HEADS, HEAD_DIM, dtype=torch.bfloat16, device=dev) for _ in "kv"]
    scd.scd_cache_read(caches[0], scd.Batch(sum(held), starts(held)), *back)
    torch.cuda.synchronize()
    return {"dense": dense, "prompt_in": first, "prompt_out": prompt, "tokens": torch.stack(tokens),
            "held": held, "back": back, "w_qkv": w_qkv, "w_out": w_out}


if __name__ == "__main__":
    out = serve()
    print("prefixes of", PREFIX, "tokens, prompts of", PROMPT, "and", STEPS, "tokens each")
    print("held:", out["held"], "generated states:", tuple(out["tokens"].shape),
          "finite:", bool(torch.isfinite(out["tokens"]).all()))
