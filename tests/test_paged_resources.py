"""Registers, LDS and scratch memory of the built kernels on a paged cache (CPU only).

The attention of many rows has two waves a SIMD and 256 registers each: one spilled
register costs a wait for every copy in flight.  The attention of few rows and the token
weights keep two workgroups of 4 waves on a CU.
"""
import os

import pytest

from test_kernel_resources import READELF, kernels


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_paged_kernels_registers_and_scratch(tmp_path):
    found = {k: v for k, v in kernels(tmp_path).items() if "paged" in k}
    for part, count, groups in (("attend_few_kernel", 16, 2), ("attend_many_kernel", 16, 1),
                                ("weights_kernel", 32, 2), ("rotary_kernel", 8, 1),
                                ("evict_", 2, 1)):
        some = {k: v for k, v in found.items() if part in k}
        assert len(some) == count, (part, len(some))
        for name, v in some.items():
            assert v["vgpr_count"] <= 256, (name, v)
            assert groups * v["group_segment_fixed_size"] <= 160 * 1024, (name, v)
            assert v["private_segment_fixed_size"] == 0, (name, v)
