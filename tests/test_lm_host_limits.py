"""Refusals of the language-model operators by their numbers alone: scales that are no numbers, layers too wide to index (host
code only, no GPU)."""
import ctypes

import pytest

from lm_util import code_of
from paper_1901_06887_b200 import binding as mt, build


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    mt.mt_shutdown()
    return mt.lib()


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf")])
def test_scales_that_are_no_numbers(lib, scale):
    desc = mt._prompt_desc(4, 1, 2, 1, 64, scale, 128, 64, 64, 64, 64, 64)
    assert lib.mt_prompt_attention(desc, None, None, None, None, None, None) == 1
    cache = ctypes.byref(mt.KvCacheDesc(2, 16, 2, 64, 16, 16, 16, 16))
    assert lib.mt_kv_attention(cache, None, 256, 64, None, 2, None, 1, 4, scale, None, None) == 1


@pytest.mark.parametrize("n", [(1 << 31) - (1 << 20), (1 << 31) - 16, (1 << 31) - 1])
def test_layers_too_wide(lib, n):
    assert code_of(mt.mt_quant_packed_bytes, 64, n, 64) == 4
    assert lib.mt_quant_pack(None, None, 1, 64, n, 64, None, None) == 4
    bank = ctypes.byref(mt.QuantBankDesc(1, 64, n, 64, 16, None))
    assert lib.mt_quant_linear(bank, None, 64, None, 1, None, n, 0, None) == 4


def test_the_widest_layer(lib):
    n = (1 << 31) - (1 << 20) - 1
    assert mt.mt_quant_packed_bytes(128, n, 64) == (n + 1) * 64 + (n + 1) * 4


def test_sizes_beyond_32_bits_are_not_cut(lib):
    for i in range(3):
        args = [64, 16, 64]
        args[i] += 1 << 32
        assert code_of(mt.mt_quant_packed_bytes, *args) == 1


def test_calls_without_a_context(lib):
    import torch
    x, i = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    assert code_of(mt.mt_prompt_attention, x, x, x, i, x) == 9
    assert code_of(mt.mt_token_logprobs, x[:, 0], i, torch.zeros(2)) == 9
    assert code_of(mt.KvCache, x, x, x, x) == 1
