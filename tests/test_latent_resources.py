"""Registers of the kernels of the latent cache, of the dense rows and of the pages: none of them spills."""
import re

import pytest

import paper_2606_07684_amd as scd
from tests.test_kernel_resources import _code_objects, _metadata


@pytest.mark.parametrize("kernel", ["latent_append_kernel", "latent_query_kernel", "latent_attend_kernel", "latent_out_kernel",
                                    "latent_expand_kernel", "rows_attend_kernel", "rows_join_kernel", "pages_reserve_kernel",
                                    "pages_copy_kernel"])
def test_no_spills(kernel):
    scd.load_library()
    with open(scd.lib_path(), "rb") as f:
        blob = f.read()
    found = {k[".name"]: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"])
             for elf in _code_objects(blob) for meta in _metadata(elf) for k in meta["amdhsa.kernels"]
             if re.search(r"\d%s" % kernel, k[".name"])}
    assert found
    assert {n: v for n, v in found.items() if v != (0, 0)} == {}
