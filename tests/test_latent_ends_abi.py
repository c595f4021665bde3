"""Sizes at the ends of what the entry points for pages take (CPU)."""
import ctypes

import pytest

import paper_2606_07684_amd as scd

UNSUP = 5
FAKE = 1 << 20  # a device address that no call reaches


@pytest.mark.parametrize("name", ["n_pages", "n_seqs", "max_pages"])
@pytest.mark.parametrize("size", [(1 << 30) + 1, (1 << 31) - 4096, (1 << 31) - 1])
def test_pools_whose_indexes_would_wrap_are_refused(name, size):
    lib = scd.load_library()
    pool = dict(n_pages=10, n_seqs=3, max_pages=4, page_tokens=16, refs=FAKE, page_table=FAKE, held=FAKE)
    pool[name] = size
    p = ctypes.byref(scd._CPages(**pool))
    moves = ctypes.byref(scd._CMoves((1 << 31) - 1, FAKE, FAKE))
    batch = ctypes.byref(scd._CBatch(pool["n_seqs"], 5, FAKE, None))
    room = 1 << 40
    assert lib.scd_pages_workspace_bytes(p) == 0
    assert lib.scd_pages_free(p, 1, FAKE, None) == UNSUP
    assert lib.scd_pages_fork(p, 1, FAKE, FAKE, None) == UNSUP
    assert lib.scd_pages_reserve(p, batch, moves, FAKE, room, None) == UNSUP
    assert lib.scd_pages_compact(p, None, moves, FAKE, room, None) == UNSUP


def test_the_largest_pool_has_a_workspace():
    lib = scd.load_library()
    p = scd._CPages(n_pages=1 << 30, n_seqs=1 << 30, max_pages=1 << 30, page_tokens=16, refs=FAKE, page_table=FAKE, held=FAKE)
    assert lib.scd_pages_workspace_bytes(ctypes.byref(p)) == 3 * 4 << 30
