"""CPU-only: numbers of entries that the 8-bit caches' kernels cannot count are refused before a launch."""
from ctypes import byref

import pytest

from tests.test_cache_host import AT, INVALID, cache, lib  # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("n", [2 ** 30 + 1, 2 ** 31 - 64, 2 ** 31 - 1])
def test_numbers_of_entries_beyond_the_kernels(lib, n):  # noqa: F811
    """With starts on the device nothing else bounds n."""
    c = cache()
    assert lib.pc_kv_quantize(byref(c), AT, None, AT, None, n, 0, AT, None, None) == INVALID
    assert lib.pc_kv_dequantize(byref(c), n, 0, None, AT, AT, None) == INVALID
    assert lib.pc_kv_dequantize(byref(c), n, 0, AT, AT, AT, None) == INVALID
