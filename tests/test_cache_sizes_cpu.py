"""Shapes of a cache whose pages could not be addressed are refused: their size in bytes would wrap (no GPU needed)."""
import ctypes as C
import os

import pytest

from paper_2601_15013_amd import binding


@pytest.mark.parametrize("layers,pages,heads,page,code", [(32, 1 << 28, 1 << 15, 256, -3), (65535, 1 << 28, 1, 256, 0), (17, 1 << 28, 16383, 256, -3),
                                                          (65535, 1 << 28, 16383, 256, -3), (16, 1 << 28, 16383, 256, 0)])
def test_bytes_beyond_63_bits(layers, pages, heads, page, code):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2601_15013_amd import build
        build.build()
    lib, n = binding.load_library(), C.c_size_t()
    cache = binding.radix_cache(layers, heads, 128, page, pages, 1, 8, 10, 0x1000, 0x1000, 0x1000, 0x1000)
    page_bytes = 2 * heads * page * 128 * 2
    assert (code == 0) == (page_bytes < 1 << 31 and layers * pages * page_bytes < 1 << 63)
    assert lib.radix_cache_bytes(C.byref(cache), C.byref(n)) == code
    if code == 0:
        assert n.value == layers * pages * page_bytes
    assert lib.radix_cache_workspace_bytes(C.byref(cache), 1, C.byref(n)) == code
