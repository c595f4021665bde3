"""What the tests of the serving operators rely on, and bounds as tight as the built kernels: which calls are prompts,
workspaces that are needed and refused, registers."""
import ctypes
import re

import pytest

from tests.test_abi import ALIGN, FAKE, NULL, OK, SHAPE, _attend, _batch, _ccache, lib  # noqa: F401
from tests.test_kernel_resources import spills  # noqa: F401
from tests.test_serving_rules import _bytes


@pytest.mark.parametrize("head_dim", [64, 128])
def test_rows_of_the_wide_scale_tests_are_prompts(head_dim):
    """8 heads over 2, 90 and 80 tokens: tiles of 256 rows, in two shares where a request may hold 432 positions.  A few
    rows' layout would need no workspace for as few, and none of this size for any."""
    args = dict(n_tokens=170, n_seqs=2, q_heads=8, kv_heads=2, head_dim=head_dim, page=16)
    tiles = 170 * 4 // 256 + 2
    assert _bytes(columns=27, **args) == 2048 + tiles * 2 * 2 * 256 * (head_dim + 2) * 4
    assert _bytes(columns=14, **args) == 0  # one share
    # three requests of 50, 60 and 40 tokens with 4 heads over 2 are a few rows: 16 of a tile, four steps at most whole
    assert _bytes(150, 3, 4, kv_heads=2, head_dim=64, page=16, columns=12) == 0


def test_a_needed_workspace_is_checked(lib):  # noqa: F811
    cache, batch = _ccache(max_pages=4096), _batch(n_tokens=1)
    need = lib.scd_cache_attend_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch._c), 4)
    # 2 heads of one tile in 32 parts each: two slots of 16 rows of 64 channels a workgroup, behind the counters
    assert need == 2048 + 2 * (2 * 32) * 16 * 66 * 4
    assert _attend(lib, cache=cache, batch=batch, ws=None)[0] == NULL
    assert _attend(lib, cache=cache, batch=batch, ws=FAKE + 8)[0] == ALIGN
    st, msg = _attend(lib, cache=cache, batch=batch, ws_bytes=need - 1)
    assert st == SHAPE and str(need) in msg
    assert _attend(lib, cache=cache, batch=_batch(n_tokens=0), ws=None, ws_bytes=0)[0] == OK


@pytest.mark.parametrize("kernel,most", [("cache_append_pages_kernel", 0), ("cache_attend_prompt_kernel", 2)])
def test_spilled_registers_are_as_few_as_built(spills, kernel, most):  # noqa: F811
    """The prompts' 2, of 128 channels, are kept from a tile's start to its chunks, outside the loop over positions."""
    got = {n: v for n, v in spills.items() if re.search(r"\d%s" % kernel, n)}
    assert got and max(got.values()) <= most, got
