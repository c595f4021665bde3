"""Infinities in keys and latents reach what the formulas say, at widths that kernels pad and at full ones."""
import pytest
import torch

import paper_2606_07684_amd as scd
from tests.latent_util import DT
from tests.test_gpu_attend_close import _latent_close, _rows_close
from tests.test_gpu_latent import Case as Latent
from tests.test_gpu_rows import Case as Rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    scd.load_library()
    yield
    torch.cuda.synchronize()


# ---- scores of -inf ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [32, 64, 96, 128, 160, 256, 288, 512])
@pytest.mark.parametrize("dr", [32, 64])
def test_latent_keys_of_minus_infinity(dtype, r, dr):
    """A shared key that makes a position's scores -inf takes it out, at every width: the same as a key so low that its
    weight is zero."""
    c = Latent(dtype, [70, 1], [3, 200], heads=2, plain=32, value=32, r=r, dr=dr, page=16)
    c.q[..., 32:] = c.q[..., 32:].abs().clamp(min=0.5)
    for channel in sorted({0, 1, dr // 2 - 1, dr // 2, dr - 8, dr - 1}):
        pages = c.pages.clone()
        both = []
        for low in (float("-inf"), -1e6):
            c.pages.copy_(pages)
            for b, p in ((0, 5), (0, 40), (0, 63), (1, 0), (1, 17), (1, 200)):
                c.pages[c.table[b][p // 16], p % 16, r + channel] = low
            both.append(c.attend())
        assert torch.isfinite(both[1]).all()
        assert torch.equal(*both), channel
        _latent_close(c, both[1])
        c.pages.copy_(pages)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("key", [32, 64, 96, 128, 160, 192])
@pytest.mark.parametrize("value", [32, 96, 128])
@pytest.mark.parametrize("stray", [0, 1])
def test_rows_keys_of_minus_infinity(dtype, key, value, stray):
    c = Rows(dtype, [100, 1, 2], [30, 300, 7], heads=4, kv_heads=2, key=key, value=value)
    c.q.copy_(c.q.abs().clamp(min=0.5))
    room = torch.zeros(*c.k.shape[:2], key + stray, dtype=DT[dtype], device="cuda")
    for channel in sorted({0, key // 2, key - 8, key - 1}):
        both = []
        for low in (float("-inf"), -1e6):
            k = room[..., :key]  # with `stray` rows that start on an element only
            k.copy_(c.k)
            for p in (0, 31, 64, 100, 129, 130, 200, 430):
                k[p, :, channel] = low
            both.append(c.attend(k=k))
        assert torch.equal(*both), channel
        kept, c.k = c.k, k
        _rows_close(c, both[1])
        c.k = kept


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,dr", [(64, 64), (96, 32), (256, 64), (512, 64)])
def test_latent_long_runs_of_minus_infinity(dtype, r, dr):
    """Blocks all of whose scores are -inf, in front of others; a request that has nothing else is left without a position;
    a query row that is not finite keeps to itself."""
    c = Latent(dtype, [3, 1, 40], [700, 300, 200], heads=5, plain=32, value=32, r=r, dr=dr, page=32)
    c.q[..., 32:] = c.q[..., 32:].abs().clamp(min=0.5)
    both = []
    for low in (float("-inf"), -1e6):
        for b, n in ((0, 400), (1, 301), (2, 130)):
            for p in range(n):
                c.pages[c.table[b][p // 32], p % 32, r + dr - 1] = low
        both.append(c.attend())
    assert torch.equal(both[0][:3], both[1][:3]) and torch.equal(both[0][4:], both[1][4:])
    assert not both[0][3].any()
    q = c.q.clone()
    q[1, 2, 3], q[30, 4, 33] = float("nan"), float("inf")
    got, clean = c.attend(q=q), both[1]
    got[1, 2] = clean[1, 2]
    got[30, 4] = clean[30, 4]
    assert torch.equal(got, torch.cat([clean[:3], got[3:4], clean[4:]]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("key,group", [(64, 1), (96, 4), (192, 4)])
def test_rows_long_runs_of_minus_infinity(dtype, key, group):
    c = Rows(dtype, [3, 1, 90], [700, 300, 200], heads=2 * group, kv_heads=2, key=key, value=64)
    c.q.copy_(c.q.abs().clamp(min=0.5))
    both, k = [], c.k.clone()
    for low in (float("-inf"), -1e6):
        for first, n in ((0, 400), (703, 301), (1004, 130)):
            k[first:first + n, :, key - 1] = low
        both.append(c.attend(k=k))
    assert torch.equal(both[0][:3], both[1][:3]) and torch.equal(both[0][4:], both[1][4:])
    assert not both[0][3].any()
    q = c.q.clone()
    q[1, 1, 3], q[30, 0, 5] = float("nan"), float("inf")
    got, clean = c.attend(q=q, k=k), both[1]
    got[1, 1] = clean[1, 1]
    got[30, 0] = clean[30, 0]
    assert torch.equal(got, torch.cat([clean[:3], got[3:4], clean[4:]]))


# ---- values that are not finite ------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,dr", [(32, 32), (96, 64), (128, 64), (160, 32), (256, 64), (288, 64), (512, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_latents_not_finite(dtype, r, dr, bad):
    """A latent that the last rows of a request attend to, and slots that none does: at every width of a latent."""
    c = Latent(dtype, [90, 1], [30, 77], heads=3, plain=32, value=64, r=r, dr=dr, page=16)
    clean = c.attend()
    c.pages[c.table[0][119 // 16], 119 % 16 + 1:] = bad                 # behind the last position
    c.pages[c.table[1][77 // 16], 77 % 16 + 1:, r - 1] = bad
    assert torch.equal(c.attend(), clean)
    for channel in (0, r // 2 + 1, r - 1):
        c.pages[c.table[0][100 // 16], 100 % 16, channel] = bad         # row 70's own position
        got = c.attend()
        assert torch.equal(got[:70], clean[:70]) and torch.equal(got[90:], clean[90:])
        assert not torch.isfinite(got[70:90]).any()
        c.pages[c.table[0][100 // 16], 100 % 16, channel] = 0.5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("key", [32, 96, 128, 192])
@pytest.mark.parametrize("value", [32, 64, 96, 128])
@pytest.mark.parametrize("tokens", [3, 150])
def test_dense_values_not_finite(dtype, key, value, tokens):
    """Of a position that the last rows attend to: their channel, and nothing else; tiles of few rows and of 128."""
    c = Rows(dtype, [tokens, 1], [70, 9], heads=4, kv_heads=2, key=key, value=value)
    clean = c.attend()
    first = tokens // 2
    for channel, bad in ((0, float("inf")), (value - 1, float("nan")), (value // 2, float("-inf"))):
        v = c.v.clone()
        v[70 + first, 1, channel] = bad
        got = c.attend(v=v)
        assert not torch.isfinite(got[first:tokens, 2:, channel]).any()
        got[first:tokens, 2:, channel] = clean[first:tokens, 2:, channel]
        assert torch.equal(got, clean)


# ---- expansion ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [32, 64, 96, 128, 160, 256, 288, 512])
def test_expand_infinities(dtype, r):
    """A latent's infinity is its products' infinity, at every width."""
    c = Latent(dtype, [70], [0], 2, 64, 32, r, 32, 16)
    k, v = (torch.empty(70, 2, d, dtype=DT[dtype], device="cuda") for d in (96, 32))
    for channel in sorted({0, r // 2, r - 8, r - 1}):
        pages = c.pages.clone()
        w_k, w_v = (torch.where(w == 0, 1.0, w).to(DT[dtype]) for w in (c.w_k, c.w_v))
        scd.scd_latent_expand(c.cache, c.batch, w_k, w_v, k, v)
        clean = k.clone(), v.clone()
        for p, x in ((0, float("inf")), (37, float("-inf")), (69, float("inf"))):
            c.pages[c.table[0][p // 16], p % 16, channel] = x
            clean[0][p, :, :64] = torch.sign(w_k[..., channel]) * x
            clean[1][p] = torch.sign(w_v[..., channel]) * x
        scd.scd_latent_expand(c.cache, c.batch, w_k, w_v, k, v)
        assert torch.equal(k, clean[0]) and torch.equal(v, clean[1]), channel
        c.pages.copy_(pages)
