"""The bound of tests/attend_error.py on the CPU: an evaluation with the kernels' roundings is inside it, and results that
lack a block of positions, count one twice, join shares by wrong weights, round weights to bf16 once, or are zero, are not."""
import numpy as np
import pytest
import torch

from tests import attend_error as E

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _pair(dtype, x):
    """fp32 x as the kernels hand it to a product: two bf16 summands, or itself."""
    if dtype == "f32":
        return x
    high = x.bfloat16().float()
    return high + (x - high).bfloat16().float()


def _attend(dtype, s, v, limit, how):
    """Weights of fp32 scores s [rows, m] in powers of two, and their sum with values v [m, channels], in fp32."""
    hidden = torch.arange(s.shape[1])[None] > limit[:, None]
    s = s.masked_fill(hidden, -torch.inf)
    top = s.amax(1, keepdim=True)
    w = torch.exp2(s - top).masked_fill(hidden, 0)
    m = s.shape[1]
    lo, hi = m // 2 // 32 * 32, m // 2 // 32 * 32 + 32
    if how == "dropped":
        w[:, lo:hi] = 0
    elif how == "twice":
        w[:, lo:hi] *= 2
    elif how == "joined":          # a share joined by the weight of a base 1/8 off
        w[:, :lo] *= 2 ** 0.125
    total = w.sum(1, keepdim=True)
    if how == "rounded":
        w = w.bfloat16().float()
    return (_pair(dtype, w) @ v) / total


LATENT = [  # lens, held, heads, plain, value, r, turned
    ([1], [332], 32, 128, 128, 256, 64), ([1], [332], 8, 64, 64, 64, 32), ([37], [100], 4, 64, 64, 96, 64),
    ([1], [20000], 2, 32, 32, 128, 32), ([6, 1], [3000, 4000], 3, 32, 32, 128, 32), ([1], [640], 4, 96, 160, 512, 64),
    ([200], [500], 2, 32, 32, 128, 32), ([1] * 4, [5000, 300, 2500, 100], 6, 32, 32, 128, 32)]
WRONG = ["dropped", "twice", "joined", "zero"]


def _latent(dtype, lens, held, heads, plain, value, r, dr, hows):
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    total = [a + b for a, b in zip(lens, held)]
    size = 16
    need = [-(-n // size) for n in total]
    table = np.full((len(lens), max(need)), -1)
    for b, n in enumerate(need):
        table[b, :n] = sum(need[:b]) + np.arange(n)
    pages = _randn(1, sum(need), size, r + dr).to(DT[dtype])
    w_k, w_v = ((_randn(i, heads, d, r) * r ** -0.5).to(DT[dtype]) for i, d in ((2, plain), (3, value)))
    q = _randn(4, cu[-1], heads, plain + dr).to(DT[dtype])
    scale = 2.0 * (plain + dr) ** -0.5
    want, off = E.latent_attend(dtype, pages.double().numpy(), table, cu, held, q.double().numpy(), w_k.double().numpy(),
                                w_v.double().numpy(), scale)
    got = {how: torch.zeros(cu[-1], heads, value, dtype=DT[dtype]) for how in hows}
    for b in range(len(lens)):
        rows = pages[torch.tensor(table[b, :need[b]])].flatten(0, 1)[:total[b]].float()
        for i in range(heads):
            x = q[cu[b]:cu[b + 1], i].float()
            a = torch.cat([_pair(dtype, x[:, :plain] @ w_k[i].float()), x[:, plain:]], 1)
            s = (a @ rows.T) * np.float32(scale * 1.4426950408889634)
            for how in hows:
                if how != "zero":
                    o = _attend(dtype, s, rows[:, :r], held[b] + torch.arange(lens[b]), how)
                    got[how][cu[b]:cu[b + 1], i] = (_pair(dtype, o) @ w_v[i].float().T).to(DT[dtype])
    return want, off, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(LATENT)))
def test_over_latents(dtype, case):
    hows = ["right"] + WRONG + (["rounded"] if dtype == "bf16" else [])
    want, off, got = _latent(dtype, *LATENT[case], hows)
    E.assert_close(got["right"].double().numpy(), want, off)
    for how in hows[1:]:
        with pytest.raises(AssertionError):
            E.assert_close(got[how].double().numpy(), want, off)


ROWS = [  # lens, pos0, heads, kv_heads, key, value
    ([1], [500], 4, 2, 128, 128), ([130], [0], 2, 1, 96, 64), ([5, 1, 300], [62, 1000, 30], 4, 1, 192, 128),
    ([1, 2, 1], [9000, 100, 4000], 4, 2, 64, 64), ([64], [64], 2, 2, 160, 96)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_over_dense_rows(dtype, case):
    lens, pos0, heads, kv_heads, key, value = ROWS[case]
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    rows = [a + b for a, b in zip(lens, pos0)]
    held_cu = np.concatenate([[0], np.cumsum(rows)]).tolist()
    q = _randn(0, cu[-1], heads, key).to(DT[dtype])
    k, v = (_randn(1, held_cu[-1], kv_heads, d).to(DT[dtype]) for d in (key, value))
    scale = 2 * key ** -0.5
    want, off = E.rows_attend(dtype, cu, pos0, held_cu, [0] * len(lens), q.double().numpy(), k.double().numpy(),
                              v.double().numpy(), scale)
    once = E.rows_attend(dtype, cu, pos0, held_cu, [0] * len(lens), q.double().numpy(), k.double().numpy(),
                         v.double().numpy(), scale, once=True)[1]
    hows = ["right"] + WRONG + (["rounded"] if dtype == "bf16" else [])
    for how in hows:
        got = torch.zeros(cu[-1], heads, value, dtype=DT[dtype])
        for b in range(len(lens)):
            for i in range(heads):
                at, held, j = slice(cu[b], cu[b + 1]), slice(held_cu[b], held_cu[b + 1]), i * kv_heads // heads
                s = (q[at, i].float() @ k[held, j].float().T) * np.float32(scale * 1.4426950408889634)
                if how != "zero":
                    got[at, i] = _attend(dtype, s, v[held, j].float(), pos0[b] + torch.arange(lens[b]), how).to(DT[dtype])
        if how == "rounded":
            E.assert_close(got.double().numpy(), want, once)
        if how == "right":
            E.assert_close(got.double().numpy(), want, off)
        else:
            for bound in (off,) if how == "rounded" else (off, once):
                with pytest.raises(AssertionError):
                    E.assert_close(got.double().numpy(), want, bound)
