"""Host side of the language-model operators: sizes and refusals that need no GPU (no compute calls)."""
import ctypes

import pytest

from lm_util import code_of
from paper_1901_06887_b200 import binding as mt, build


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    mt.mt_shutdown()
    return mt.lib()


def test_packed_bytes(lib):
    # half a byte per weight and two bytes per scale, outputs rounded up to tiles of 16
    for k, n, g in ((64, 1, 32), (64, 16, 64), (4096, 4096, 64), (384, 17, 128), (8192, 50, 8192)):
        rows = -(-n // 16) * 16
        assert mt.mt_quant_packed_bytes(k, n, g) == rows * (k // 2) + rows * (k // g) * 2
    for args, code in (((0, 4, 64), 1), ((64, 0, 64), 1), ((64, 4, 0), 1), ((96, 4, 32), 4), ((128, 4, 16), 4), ((192, 4, 96), 4),
                       ((128, 4, 256), 4), ((1 << 22, 4, 64), 4)):
        assert code_of(mt.mt_quant_packed_bytes, *args) == code
    assert lib.mt_quant_packed_bytes(64, 4, 64, None) == 1


def prompt(**kw):
    d = dict(n=4, seqs=1, hq=2, hk=1, dim=64, scale=0.125, strides=(128, 64, 64, 64, 64, 64))
    d.update(kw)
    return mt._prompt_desc(d["n"], d["seqs"], d["hq"], d["hk"], d["dim"], d["scale"], *d["strides"])


def test_prompt_refusals(lib):
    f = lambda desc: lib.mt_prompt_attention(desc, None, None, None, None, None, None)
    assert f(None) == 1
    for kw, code in ((dict(n=-1), 1), (dict(seqs=-1), 1), (dict(hq=0), 1), (dict(hk=0), 1), (dict(dim=96), 4), (dict(hq=3, hk=2), 4),
                     (dict(n=(1 << 30) + 1), 4), (dict(strides=(128, 64, 64, 64, 64, 60)), 4), (dict(strides=(128, 63, 64, 64, 64, 64)), 4),
                     (dict(strides=(0, 64, 64, 64, 64, 64)), 4), (dict(strides=(1 << 36, 64, 64, 64, 64, 64)), 4), (dict(), 9)):
        assert f(prompt(**kw)) == code, kw


def cache(**kw):
    d = dict(pages=2, page=16, heads=2, dim=64, p=(16, 16, 16, 16))
    d.update(kw)
    return ctypes.byref(mt.KvCacheDesc(d["pages"], d["page"], d["heads"], d["dim"], *d["p"]))


def test_cache_refusals(lib):
    append = lambda c, s=(128, 64, 128, 64), n=1: lib.mt_kv_append(c, None, s[0], s[1], None, s[2], s[3], None, n, None)
    read = lambda c, n=1: lib.mt_kv_read(c, None, n, None, None, None)
    attend = lambda c, q=(256, 64), width=2, n=1, heads=4: lib.mt_kv_attention(c, None, q[0], q[1], None, width, None, n, heads, 0.125, None, None)
    for f in (append, read, attend):
        assert f(None) == 1
        for kw, code in ((dict(pages=-1), 1), (dict(heads=0), 1), (dict(dim=80), 4), (dict(page=48), 4), (dict(page=8), 4), (dict(page=512), 4),
                         (dict(p=(16, None, 16, 16)), 1), (dict(p=(16, 16, 8, 16)), 1), (dict(), 9)):
            assert f(cache(**kw)) == code, kw
        assert f(cache(), n=-1) == 1
    assert append(cache(), (128, 60, 128, 64)) == 4
    assert attend(cache(), heads=3) == 4 and attend(cache(), heads=34) == 4 and attend(cache(), heads=0) == 1
    assert attend(cache(), width=-1) == 1 and attend(cache(), width=1 << 27) == 4 and attend(cache(), q=(256, 4)) == 4
    assert attend(cache(), n=1 << 19) == 4


def test_linear_and_logprob_refusals(lib):
    bank = lambda *a: ctypes.byref(mt.QuantBankDesc(*a, 16, None))
    f = lambda b, xs=128, n=1, ys=8, dt=0: lib.mt_quant_linear(b, None, xs, None, n, None, ys, dt, None)
    assert f(None) == 1 and f(bank(0, 128, 8, 64)) == 1 and f(bank(2, 128, 8, 48)) == 4 and f(bank(2, 100, 8, 50)) == 4
    good = bank(2, 128, 8, 64)
    assert f(good, xs=127) == 4 and f(good, n=-1) == 1 and f(good, dt=2) == 1 and f(good, n=2, ys=7) == 1 and f(good) == 9
    g = lambda dt=0, stride=100, n=1, vocab=100, top=0: lib.mt_token_logprobs(None, dt, stride, n, vocab, None, top, None, None, None, None, None)
    assert g(dt=2) == 1 and g(n=-1) == 1 and g(vocab=0) == 1 and g(top=-1) == 1 and g(top=33) == 4 and g(vocab=1 << 30) == 4
    assert g(stride=-1) == 4 and g() == 9
    assert lib.mt_quant_pack(None, None, 1, 128, 8, 64, None, None) == 9 and lib.mt_quant_pack(None, None, -1, 128, 8, 64, None, None) == 1
