"""How many places a call of the book of pages may have (host checks; no GPU): the kernels' counters are 32 bits wide and step past the last place."""
import ctypes

import pytest

from paper_1901_06887_b200 import binding as mt, build

MOST = 1 << 30
NOT_INIT = 9


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    mt.mt_shutdown()
    return mt.lib()


def calls(lib, n, rows=3):
    b = ctypes.byref(mt.KvPagesDesc(8, 16, rows, 4, 16, 4, 4))
    cache = (ctypes.POINTER(mt.KvCacheDesc) * 1)(ctypes.pointer(mt.KvCacheDesc(2, 16, 2, 64, 16, 16, 16, 16)))
    return [lib.mt_kv_reserve(b, None, None, n, None, 0, None), lib.mt_kv_fork(b, None, None, n, None, None), lib.mt_kv_release(b, None, n, None),
            lib.mt_kv_compact(b, None, n, None)], lib.mt_kv_copy(cache, 1, None, n, None)


def test_places(lib):
    for n, code in ((-1, 1), (1, NOT_INIT), (MOST, NOT_INIT), (MOST + 1, 4), (2 ** 31 - 1, 4)):
        assert calls(lib, n) == ([code] * 4, code), n


def test_rows(lib):
    for rows, code in ((MOST, NOT_INIT), (MOST + 1, 4), (2 ** 31 - 1, 4)):
        assert calls(lib, 1, rows)[0] == [code] * 4, rows
