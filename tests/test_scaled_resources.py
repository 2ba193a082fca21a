"""Registers and scratch memory of the kernels of the 8-bit path, from the metadata of the built library (no GPU needed)."""
import re

import pytest

from test_kernel_resources import _waves, kernels  # noqa: F401


@pytest.mark.parametrize("pattern,waves", [
    (r"k_scaled_tiles<.*>", 2),                                                    # eight wavefronts, a compute unit's LDS
    (r"k_scaled_stream<false, 1, 1, 2, .*>", 4), (r"k_scaled_stream<true, 1, 1, 2, .*>", 4),
    (r"k_scaled_stream<false, 2, 2, 1, .*>", 4), (r"k_scaled_stream<true, 2, 1, 2, .*>", 2), (r"k_scaled_stream<true, 2, 2, 1, .*>", 2),
    (r"k_rows<unsigned short, 4, 4>", 8), (r"k_scaled_combine<.*>", 8),
])
def test_wavefronts_per_simd(kernels, pattern, waves):  # noqa: F811
    """As many wavefronts as the workgroup shapes are made for, none by way of scratch memory."""
    mine = {n: k for n, k in kernels.items() if re.fullmatch(pattern, n)}
    assert mine
    for name, k in mine.items():
        assert _waves(k) >= waves, (name, k[".vgpr_count"])
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, name
