"""The paged cache's descriptions at their limits and when they change, without a GPU."""
import ctypes

import pytest

from paper_2608_01150_b200 import binding as B
from test_cache_calls import CUDA, INVALID, batch_desc, cache_desc, no_device


# ---------------------------------------------------------------------------------------------- limits
@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("name", ["page_stride", "token_stride", "head_stride"])
def test_strides_fit_32_bits_in_units_of_16_bytes(fmt, name):
    """2^35 bf16 elements are 2^32 such units: none of them is left in 32 bits."""
    lib, b = B.lib(), batch_desc()
    scales = dict(k_scale=4096, v_scale=4096) if fmt else {}
    c = cache_desc(format=fmt, **scales, **{name: 1 << 35})
    assert lib.zl_cache_write(ctypes.byref(c), ctypes.byref(b), 4096, 4096, 128, 0) == INVALID


@no_device
@pytest.mark.parametrize("name", ["page_stride", "token_stride", "head_stride"])
def test_the_largest_strides_are_taken(name):
    lib, c, b = B.lib(), cache_desc(**{name: (1 << 35) - 8}), batch_desc()
    assert lib.zl_cache_write(ctypes.byref(c), ctypes.byref(b), 4096, 4096, 128, 0) == CUDA
