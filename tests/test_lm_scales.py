"""Scales of cross attention at the ends of their range (host checks; no GPU): powers of two are taken of scores times scale log2(e), which has to be a number."""
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


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scales_that_pass_the_largest_number(lib, sign):
    def code(scale):
        return lib.mt_cross_attention(mt._cross_desc(4, 9, 1, 2, 1, 64, sign * scale, 128, 64, 64, 64, 64, 64), *[None] * 7)
    for scale in (LARGEST, 2.4e38, math.inf):
        assert code(scale) == 1, scale
    for scale in (2.35e38, 1.0, 1e-45, 0.0):
        assert code(scale) == NOT_INIT, scale
