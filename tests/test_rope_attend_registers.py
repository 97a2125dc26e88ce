"""Registers of the kernels of spla_rotate, spla_append_rope and spla_attend: nothing is spilled,
and each kernel stays within what its count of wavefronts per SIMD leaves (512 registers)."""

import re

import pytest

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


@pytest.mark.parametrize("pattern,count,vgprs", [
    (r"rotate_(any_)?kernel<", 12, 128),
    (r"append_rope_one_kernel<", 4, 64),
    (r"append_fused_kernel<128, (true|false)>", 2, 256),
    (r"attend_stream_kernel<", 4, 256),
    (r"attend_rows_kernel<", 2, 256),
    (r"attend_tile_kernel<\d+, \d>", 8, 168),
    (r"attend_join_kernel<", 4, 128),
])
def test_no_spills(kernels, pattern, count, vgprs):  # noqa: F811
    hit = {n: k for n, k in kernels.items() if re.match(pattern, n)}
    assert len(hit) == count, sorted(hit)
    for n, k in hit.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
        assert k[".vgpr_count"] <= vgprs, (n, k[".vgpr_count"])
