"""Refusals of token sampling, rotary positions, the book of a cache's pages and cross attention that need no GPU (no compute calls)."""
import ctypes

import pytest

from paper_1901_06887_b200 import binding as mt, build


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    mt.mt_shutdown()
    return mt.lib()


def test_cross_refusals(lib):
    base = dict(n=4, m=9, seqs=1, hq=2, hk=1, dim=64, scale=0.125, strides=(128, 64, 64, 64, 64, 64))

    def f(**kw):
        d = {**base, **kw}
        return lib.mt_cross_attention(mt._cross_desc(d["n"], d["m"], d["seqs"], d["hq"], d["hk"], d["dim"], d["scale"], *d["strides"]),
                                      None, None, None, None, None, None, None)
    assert lib.mt_cross_attention(None, None, None, None, None, None, None, None) == 1
    for kw, code in ((dict(n=-1), 1), (dict(m=-1), 1), (dict(seqs=-1), 1), (dict(hq=0), 1), (dict(hk=0), 1), (dict(dim=96), 4), (dict(hq=3, hk=2), 4),
                     (dict(n=(1 << 30) + 1), 4), (dict(m=(1 << 30) + 1), 4), (dict(strides=(128, 64, 64, 64, 64, 60)), 4), (dict(scale=float("nan")), 1),
                     (dict(scale=float("inf")), 1), (dict(strides=(0, 64, 64, 64, 64, 64)), 4), (dict(strides=(1 << 36, 64, 64, 64, 64, 64)), 4), (dict(), 9)):
        assert f(**kw) == code, kw


def test_rotate_refusals(lib):
    base = dict(n=4, heads=2, dim=64, rotary=64, axes=1, sections=(32, 0, 0, 0), dtype=0, strides=(128, 64, 128, 64))

    def f(**kw):
        d = {**base, **kw}
        return lib.mt_rotate(mt._rotate_desc(d["n"], d["heads"], d["dim"], d["rotary"], d["axes"], *d["sections"], 0, 0, d["dtype"], *d["strides"]),
                             None, None, None, None, None)
    assert lib.mt_rotate(None, None, None, None, None, None) == 1
    for kw, code in ((dict(n=-1), 1), (dict(heads=0), 1), (dict(dim=0), 1), (dict(rotary=0), 1), (dict(dtype=2), 1), (dict(axes=0), 1), (dict(axes=5), 1),
                     (dict(sections=(31, 0, 0, 0)), 1), (dict(sections=(40, -8, 0, 0), axes=2), 1), (dict(rotary=80, sections=(40, 0, 0, 0)), 1),
                     (dict(dim=60), 1), (dict(dim=68), 4), (dict(dim=520), 4), (dict(rotary=24, sections=(12, 0, 0, 0)), 4), (dict(heads=65536), 4),
                     (dict(strides=(128, 60, 128, 64)), 4), (dict(strides=(128, -64, 128, 64)), 4), (dict(strides=(1 << 36, 64, 128, 64)), 4),
                     (dict(strides=(128, 64, 0, 64)), 1), (dict(strides=(128, 64, 128, 56)), 1), (dict(), 9)):
        assert f(**kw) == code, kw


def book(**kw):
    d = dict(pages=8, page=16, rows=3, width=4, p=(16, 4, 4))
    d.update(kw)
    return ctypes.byref(mt.KvPagesDesc(d["pages"], d["page"], d["rows"], d["width"], *d["p"]))


def test_page_refusals(lib):
    calls = (lambda b, n=1: lib.mt_kv_reserve(b, None, None, n, None, 0, None), lambda b, n=1: lib.mt_kv_fork(b, None, None, n, None, None),
             lambda b, n=1: lib.mt_kv_release(b, None, n, None), lambda b, n=1: lib.mt_kv_compact(b, None, n, None))
    for f in calls:
        assert f(None) == 1
        for kw, code in ((dict(pages=-1), 1), (dict(rows=-1), 1), (dict(width=-1), 1), (dict(page=48), 4), (dict(page=8), 4), (dict(page=512), 4),
                         (dict(width=1 << 27), 4), (dict(pages=2 ** 31 - 1), 4), (dict(p=(None, 4, 4)), 1), (dict(p=(16, None, 4)), 1), (dict(p=(16, 4, None)), 1),
                         (dict(p=(8, 4, 4)), 1), (dict(p=(16, 2, 4)), 1), (dict(), 9)):
            assert f(book(**kw)) == code, kw
        assert f(book(), -1) == 1
    assert lib.mt_kv_reserve(book(), None, None, 1, None, -1, None) == 1


def test_copy_refusals(lib):
    def f(*caches, n=1):
        descs = [mt.KvCacheDesc(*c, 16, 16, 16, 16) for c in caches]
        array = (ctypes.POINTER(mt.KvCacheDesc) * max(1, len(descs)))(*[ctypes.pointer(d) for d in descs])
        return lib.mt_kv_copy(array, len(descs), None, n, None)
    good = (2, 16, 2, 64)
    assert f(good, n=-1) == 1 and lib.mt_kv_copy(None, -1, None, 1, None) == 1 and lib.mt_kv_copy(None, 1, None, 1, None) == 1
    assert f((2, 48, 2, 64)) == 4 and f((2, 16, 0, 64)) == 1 and f((2, 16, 2, 96)) == 4
    assert f(good, (3, 16, 2, 64)) == 1 and f(good, (2, 32, 2, 64)) == 1
    assert lib.mt_kv_copy((ctypes.POINTER(mt.KvCacheDesc) * 1)(), 1, None, 1, None) == 1
    assert f(good) == 9 and f(good, (2, 16, 3, 128)) == 9


def test_sample_refusals(lib):
    f = lambda dt=0, stride=100, n=1, vocab=100: lib.mt_token_sample(None, dt, stride, n, vocab, *[None] * 8)
    assert f(dt=2) == 1 and f(n=-1) == 1 and f(vocab=0) == 1 and f(vocab=1 << 30) == 4 and f(n=(1 << 29) + 1) == 4 and f(stride=-1) == 4 and f(stride=1 << 36) == 4 and f() == 9
