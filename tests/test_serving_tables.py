"""The binding refuses a table of turns that does not hold what the library reads from it."""
import ctypes

import pytest
import torch

import paper_2606_07684_amd as scd


def _rotary():
    return scd.Rotary(64, 1e4, rotary_dim=32)


class _Device:
    """The two calls that the binding makes of a device buffer's size and place, without a device."""
    def __new__(cls, nbytes):
        t = torch.empty(nbytes, dtype=torch.uint8)
        t.__class__ = type("DeviceBytes", (torch.Tensor,), {"is_cuda": True})
        return t


def test_table_must_be_device_memory():
    r = _rotary()
    need = int(scd.load_library().scd_rotary_table_bytes(ctypes.byref(r._c), 100))
    assert need == 100 * 16 * 8
    with pytest.raises(ValueError, match="CUDA"):
        scd._turns_args(scd.RotaryTable(torch.empty(need, dtype=torch.uint8), 100, r))


@pytest.mark.parametrize("nbytes,positions,fits", [(12800, 100, True), (12799, 100, False), (12800, 101, False),
                                                   (12800, 1, True), (12800, 0, False), (0, 100, False)])
def test_table_must_hold_its_positions(nbytes, positions, fits):
    table = scd.RotaryTable(_Device(nbytes), positions, _rotary())
    if fits:
        assert scd._turns_args(table)[2] == positions
    else:
        with pytest.raises(ValueError, match="rotary table holds"):
            scd._turns_args(table)


@pytest.mark.gpu
def test_calls_refuse_a_short_table():
    r = _rotary()
    table = scd.scd_rotary_table(r, 100)
    x = torch.zeros(3, 2, 64, device="cuda")
    batch = scd.Batch(3)
    cache = scd.PagedCache(*[torch.zeros(1, 2, 16, 64, dtype=torch.int8, device="cuda") for _ in "kv"],
                           *[torch.zeros(1, 2, device="cuda") for _ in "kv"],
                           torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
    for bad in (scd.RotaryTable(table.buffer, 101, r), scd.RotaryTable(table.buffer[:-8], 100, r),
                scd.RotaryTable(table.buffer, 100, scd.Rotary(64, 1e4)), scd.RotaryTable(table.buffer.cpu(), 100, r)):
        with pytest.raises(ValueError, match="rotary table"):
            scd.scd_rotary(bad, batch, x, None, x, None)
        with pytest.raises(ValueError, match="rotary table"):
            scd.scd_cache_append(cache, batch, x, x, bad)
    scd.scd_rotary(table, batch, x, None, x, None)
    scd.scd_cache_append(cache, batch, x, x, table)
