"""Tensors of a shape that the binding has to refuse before it reads their sizes (no GPU: nothing gets as far as the library)."""
import pytest
import torch

from paper_1901_06887_b200 import binding as mt


@pytest.mark.parametrize("shape", [(), (4, 1, 1), (1, 4), (5,), (3,)])
def test_positions(monkeypatch, shape):
    monkeypatch.setattr(mt, "_device", -1)                      # (where tensors of the host say they are)
    monkeypatch.setattr(mt, "_lib", object())
    x = torch.zeros((4, 2, 64))
    with pytest.raises(mt.MtError) as e:
        mt.mt_rotate(x, torch.zeros(shape, dtype=torch.int32), torch.zeros(32), x, stream=0)
    assert e.value.code == 1
