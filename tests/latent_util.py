"""Inputs and bounds that the tests of the latent cache and of attention over dense rows share."""
import numpy as np
import torch

import paper_2606_07684_amd as scd

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # one rounding to the type is off by at most this times the value


def f64(t):
    return t.double().cpu().numpy()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def batch_of(lens, held, tokens=None):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()
    return scd.Batch(cu[-1] if tokens is None else tokens, ints(cu), None if held is None else ints(held)), cu


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def strided(x, how):
    """x's values behind other strides."""
    t, h, d = x.shape
    if how == "dense":
        return x.clone()
    if how == "fused":     # heads of a wider row
        y = torch.zeros(t, h + 3, d, dtype=x.dtype, device=x.device)[:, 2:2 + h]
    elif how == "heads_first":
        y = torch.zeros(h, t, d, dtype=x.dtype, device=x.device).transpose(0, 1)
    elif how == "odd":     # rows that start on an element only
        y = torch.zeros(t * h * (d + 1) + 1, dtype=x.dtype, device=x.device)[1:].view(t, h, d + 1)[..., :d]
    y.copy_(x)
    return y


def paged(lens, size, seed, spare=3, cols=None):
    """Pages in scattered order for requests that hold `lens` tokens: a table (list of rows), number of pages."""
    need = [-(-n // size) for n in lens]
    n_pages = sum(need) + spare
    order = np.random.default_rng(seed).permutation(n_pages).tolist()
    cols = cols or max(1, max(need))
    table = []
    for n in need:
        row = [order.pop() for _ in range(n)]
        table.append((row + [-1] * cols)[:cols])
    return table, n_pages


def attend_bound(dtype, want, mass, loud, terms):
    """How far a result may be off: one rounding of it; weights off by what their scores are, twice (in the weight
    and in the sum), and rounded once (bf16); sums of `terms` products in fp32.  `mass` is what the magnitudes of
    a result's terms add up to, `loud` a score's.  Queries and weighted latents as two bf16 summands are off by
    2^-16 at most.  fp32 exponentials are within 2^-22."""
    score = loud * ((2.0 ** -16 if dtype == "bf16" else 0.0) + terms * 2.0 ** -24)
    weight = 2 * (np.exp(score) - 1) + 2.0 ** -21 + (2.0 ** -8 + 2.0 ** -16 if dtype == "bf16" else 0.0)
    return 1.01 * HALF[dtype] * np.abs(want) + mass * (weight + terms * 2.0 ** -24) + 1e-30
