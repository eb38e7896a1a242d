"""Caches, banks and books of pages that were put together for another GPU than the context's, before there was a context or for an earlier one: refused, before
the library sees them.  No GPU: what a call would hand to the library is only counted, and tensors say where they lie."""
import pytest
import torch

from paper_1901_06887_b200 import binding as mt

BF16, I32, I64, U8, F32 = torch.bfloat16, torch.int32, torch.int64, torch.uint8, torch.float32


class On:
    """A tensor that says it lies on a GPU."""
    is_cuda = True

    def __init__(self, device, *shape, dtype):
        self.t, self.at = torch.zeros(shape, dtype=dtype), device

    def get_device(self):
        return self.at

    def __getattr__(self, name):
        return getattr(self.t, name)


class Library:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


def handles(device, monkeypatch):
    """Put together with no context."""
    monkeypatch.setattr(mt, "_device", None)
    z = lambda *s, dtype: On(device, *s, dtype=dtype)
    cache = mt.KvCache(z(2, 1, 16, 32, dtype=U8), z(2, 1, 16, 2, dtype=BF16), z(2, 1, 16, 32, dtype=U8), z(2, 1, 16, 2, dtype=BF16))
    pages = mt.KvPages(z(2, dtype=I32), z(3, 2, dtype=I32), z(3, dtype=I32), 16)
    bank = object.__new__(mt.QuantBank)                         # (its constructor allocates on the GPU)
    bank.in_features, bank.out_features, bank.device, bank.ref = 64, 8, device, None
    return cache, pages, bank


def calls(cache, pages, bank, at):
    z = lambda *s, dtype: On(at, *s, dtype=dtype)
    rows, heads = z(3, dtype=I32), z(3, 1, 64, dtype=BF16)
    return {
        "append": lambda: mt.mt_kv_append(cache, heads, heads, z(3, dtype=I64), stream=0),
        "read": lambda: mt.mt_kv_read(cache, z(3, dtype=I64), heads, heads, stream=0),
        "attention": lambda: mt.mt_kv_attention(cache, heads, z(3, 2, dtype=I32), rows, heads, stream=0),
        "linear": lambda: mt.mt_quant_linear(z(3, 64, dtype=BF16), rows, bank, z(3, 8, dtype=F32), stream=0),
        "reserve": lambda: mt.mt_kv_reserve(pages, rows, rows, z(3, dtype=I64), stream=0),
        "fork": lambda: mt.mt_kv_fork(pages, rows, rows, z(3, 3, dtype=I32), stream=0),
        "release": lambda: mt.mt_kv_release(pages, rows, stream=0),
        "compact": lambda: mt.mt_kv_compact(pages, z(3, 3, dtype=I32), stream=0),
        "copy": lambda: mt.mt_kv_copy(mt.KvCopier([cache]), z(3, 3, dtype=I32), stream=0),
    }


@pytest.mark.parametrize("name", ["append", "read", "attention", "linear", "reserve", "fork", "release", "compact", "copy"])
@pytest.mark.parametrize("made_for,context", [(1, 0), (0, 1), (0, 0), (1, 1)])
def test_made_for_another_gpu(monkeypatch, made_for, context, name):
    made = handles(made_for, monkeypatch)
    library = Library()
    monkeypatch.setattr(mt, "_lib", library)
    monkeypatch.setattr(mt, "_device", context)
    call = calls(*made, context)[name]
    if made_for == context:
        call()
        assert library.calls == 1
    else:
        with pytest.raises(mt.MtError) as e:
            call()
        assert e.value.code == 1 and library.calls == 0


def test_caches_of_two_gpus(monkeypatch):
    one, two = handles(0, monkeypatch)[0], handles(1, monkeypatch)[0]
    monkeypatch.setattr(mt, "_lib", Library())
    for context in (0, 1):
        monkeypatch.setattr(mt, "_device", context)
        with pytest.raises(mt.MtError) as e:
            mt.mt_kv_copy(mt.KvCopier([one, two]), On(context, 3, 3, dtype=I32), stream=0)
        assert e.value.code == 1
