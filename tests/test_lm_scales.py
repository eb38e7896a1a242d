"""Scales of attention at the ends of their range (host checks; no GPU).  Products are taken in powers of two, with scale log2(e): that has to be a number."""
import ctypes
import math

import pytest

from paper_1901_06887_b200 import binding as mt, build

LARGEST = 3.4028234663852886e38
NOT_INIT = 9


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    mt.mt_shutdown()
    return mt.lib()


def codes(lib, scale):
    prompt = mt._prompt_desc(4, 1, 2, 1, 64, scale, 128, 64, 64, 64, 64, 64)
    cross = mt._cross_desc(4, 9, 1, 2, 1, 64, scale, 128, 64, 64, 64, 64, 64)
    cache = ctypes.byref(mt.KvCacheDesc(2, 16, 2, 64, 16, 16, 16, 16))
    return {lib.mt_prompt_attention(prompt, None, None, None, None, None, None),
            lib.mt_cross_attention(cross, None, None, None, None, None, None, None),
            lib.mt_kv_attention(cache, None, 256, 64, None, 2, None, 1, 4, scale, None, None)}


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scales_that_pass_the_largest_number(lib, sign):
    for scale in (LARGEST, 2.4e38, math.inf):
        assert codes(lib, sign * scale) == {1}, scale
    for scale in (2.3e38, 1.0, 1e-45, 0.0):
        assert codes(lib, sign * scale) == {NOT_INIT}, scale
