"""Rules of the serving operators that need no GPU: what a call's workspace holds by its arguments, and the registers
of the built kernels."""
import ctypes
import re

import pytest

import paper_2606_07684_amd as scd
from tests.test_kernel_resources import spills  # noqa: F401

FAKE = 0x7f0000000000


def _bytes(n_tokens, n_seqs, q_heads, kv_heads=8, head_dim=128, page=64, columns=128):
    cache = scd._CCache(1000, page, kv_heads, head_dim, columns, *[FAKE] * 5)
    batch = scd.Batch(n_tokens)
    batch._c.n_seqs, batch._c.cu_seqlens = n_seqs, FAKE
    return scd.load_library().scd_cache_attend_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch._c), q_heads)


@pytest.mark.parametrize("args,want", [
    # one token of a request whose table holds 512 positions: four steps at most, segments stay whole
    (dict(n_tokens=1, n_seqs=1, q_heads=32, columns=8), 0),
    # one more column: 8 segments in 9 .. steps: two slots of 16 rows for each of the workgroups
    (dict(n_tokens=1, n_seqs=1, q_heads=32, columns=9), 2048 + 2 * (8 * 5) * 16 * 130 * 4),
    # a long table: 32 parts of each segment, or as many workgroups as a launch has
    (dict(n_tokens=1, n_seqs=1, q_heads=32, columns=512), 2048 + 2 * (8 * 32) * 16 * 130 * 4),
    (dict(n_tokens=64, n_seqs=64, q_heads=32, columns=512), 2048 + 2 * 512 * 16 * 130 * 4),
    (dict(n_tokens=0, n_seqs=1, q_heads=32), 0)])
def test_workspace_of_a_few_rows(args, want):
    assert _bytes(**args) == want


def test_workspace_of_prompts_covers_both_types():
    """4096 tokens of one request: 65 tiles of 256 rows over 8 heads need no shares in bf16; fp32 rows need slots.
    One size serves either."""
    assert _bytes(4096, 1, 32) == 2048 + 2 * 512 * 16 * 130 * 4
    # 64 tokens behind a long prefix: 2 tiles x 8 heads in 16 shares of 256 rows
    assert _bytes(64, 1, 32) == 2048 + 2 * 8 * 16 * 256 * 130 * 4


@pytest.mark.parametrize("kernel,most", [
    ("cache_attend_rows_kernel", 0), ("cache_attend_prompt_kernel", 8), ("cache_attend_join_kernel", 0),
    ("cache_append_few_kernel", 0), ("cache_append_pages_kernel", 8), ("cache_read_kernel", 0), ("rotary_kernel", 0)])
def test_spilled_registers(spills, kernel, most):  # noqa: F811
    got = {n: v for n, v in spills.items() if re.search(r"\d%s" % kernel, n)}
    assert got
    assert {n: v for n, v in got.items() if v > most} == {}
