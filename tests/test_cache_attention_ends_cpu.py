"""What the calls on 4-bit caches refuse at the ends of their arguments, on a machine without a GPU."""
import ctypes

import pytest

from paper_2510_26527_b200 import binding, buildlib

FAKE = 0x1000           # aligned, never dereferenced on the host
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    buildlib.build()
    return binding.load_library()


@pytest.mark.parametrize("scale", [1.1e30, -1.1e30, 3e38, -3e38, float("inf"), float("-inf"), float("nan")])
def test_attention_and_weights_refuse_scales_past_1e30(lib, scale):
    """scale * log2(e), and its product with a query, would leave fp32."""
    s = ctypes.byref(binding.CachePagesStruct(4, 8, 100, 16, FAKE, FAKE, FAKE, FAKE))
    r = ctypes.byref(binding.BlockRows(FAKE, None, FAKE, None, 20))
    assert lib.polyspec_cache_attention(s, r, FAKE, 1024, 8, 4, 128, scale, FAKE, FAKE, None, None, FAKE, BIG, None) == binding.ERR_INVALID_ARG
    assert lib.polyspec_cache_weigh(s, r, FAKE, 1024, 8, 4, 128, scale, FAKE, FAKE, 1.0, FAKE, None, None) == binding.ERR_INVALID_ARG
