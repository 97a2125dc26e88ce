"""Registers of the kernels of the 8-bit cache and of the per-head norms: each stays within what
its count of workgroups per compute unit leaves (512 registers per SIMD), and none but the tiles
of 128 rows, whose masks' bounds may lie in scratch memory, spills any."""

import re

import pytest

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


@pytest.mark.parametrize("pattern,count,vgprs,spills", [
    (r"norm_rotate_kernel<", 12, 64, 0),
    (r"norm_rotate_grad_kernel<", 8, 168, 0),
    (r"append8_kernel<", 12, 168, 0),
    (r"read8_kernel<", 4, 64, 0),
    (r"attend8_stream_kernel<", 4, 168, 0),
    (r"attend8_tile_kernel<float", 8, 256, 1),
    (r"attend8_tile_kernel<spla::bf16_t, 64", 8, 168, 0),
    (r"attend8_tile_kernel<spla::bf16_t, 128, [01], true", 2, 168, 4),
    (r"attend8_tile_kernel<spla::bf16_t, 128, [23], true", 2, 256, 0),
    (r"attend8_tile_kernel<spla::bf16_t, 128, [0-2], false", 3, 168, 6),
    (r"attend8_tile_kernel<spla::bf16_t, 128, 3, false", 1, 256, 0),
])
def test_registers(kernels, pattern, count, vgprs, spills):  # noqa: F811
    hit = {n: k for n, k in kernels.items() if re.match(pattern, n)}
    assert len(hit) == count, sorted(hit)
    for n, k in hit.items():
        assert k[".vgpr_spill_count"] <= spills, n
        assert k[".private_segment_fixed_size"] <= (4 * spills + 4 if spills else 0), n
        assert k[".vgpr_count"] <= vgprs, (n, k[".vgpr_count"])
