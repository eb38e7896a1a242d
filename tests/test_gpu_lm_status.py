"""The sticky status of the operators of language-model tenants: code and index come from one error of one call."""
import numpy as np
import pytest
import torch

from lm_util import init, random_cache
from paper_1901_06887_b200 import binding as mt, synth

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Ops:
    """Calls that go wrong at a chosen index."""

    def __init__(self):
        init()
        g = torch.Generator(device="cuda").manual_seed(0)
        self.bank = mt.QuantBank(torch.zeros((2, 8, 32), dtype=torch.uint8, device="cuda"), torch.ones((2, 8, 1), dtype=torch.bfloat16, device="cuda"))
        self.cache = random_cache(4, 16, 1, 64, g)
        self.rows = torch.zeros((400, 1, 64), dtype=torch.bfloat16, device="cuda")

    def linear(self, bad):
        ids = i32([0] * 400)
        ids[bad] = 5
        mt.mt_quant_linear(self.rows[:, 0], ids, self.bank, torch.empty((400, 8), device="cuda"))

    def attention(self, bad):
        tables = i32([[0]] * 8)
        tables[bad] = 9
        mt.mt_kv_attention(self.cache, self.rows[:8], tables, i32([3] * 8), torch.empty_like(self.rows[:8]))

    def append(self, bad):
        slots = torch.full((50,), -1, device="cuda")
        slots[bad] = 1000
        mt.mt_kv_append(self.cache, self.rows[:50], self.rows[:50], slots)

    def prompt(self, bad):
        offsets = i32([10 * i for i in range(9)])
        offsets[bad + 1] = 0 if bad else -1
        mt.mt_prompt_attention(self.rows[:80], self.rows[:80], self.rows[:80], offsets, torch.empty_like(self.rows[:80]))


def test_two_errors_between_two_reads():
    ops = Ops()
    ops.linear(300)
    ops.attention(1)
    assert mt.mt_get_async_status() == (2, 300)                  # (bad id, row): sequence 1 is the second call's
    ops.attention(5)
    ops.linear(2)
    assert mt.mt_get_async_status() == (1, 5)
    assert mt.mt_get_async_status() == (0, -1)


def test_the_first_call_counts_also_where_the_kind_is_the_same():
    ops = Ops()
    ops.append(40)
    ops.attention(3)
    ops.prompt(2)
    assert mt.mt_get_async_status() == (1, 40)
    ops.prompt(6)
    ops.append(0)
    assert mt.mt_get_async_status() == (1, 6)
    assert mt.mt_get_async_status() == (0, -1)


def test_the_smallest_index_of_a_call():
    ops = Ops()
    ops.append([7, 30, 49])
    assert mt.mt_get_async_status() == (1, 7)
    ops.linear([399, 256, 310])                                  # in the second launch of the call
    assert mt.mt_get_async_status() == (2, 256)
    ops.linear([399, 20])                                        # in both
    assert mt.mt_get_async_status() == (2, 20)


def test_beside_an_error_of_a_batch():
    wl = synth.make_workload(1)
    mt.mt_shutdown()
    mt.mt_init(0, 64, wl.n)
    try:
        for m in wl.models:
            mt.mt_register_model(m)
        ops = Ops()
        x = torch.from_numpy(wl.inputs.view(np.int16)).cuda().view(torch.bfloat16)
        ids = torch.from_numpy(wl.model_ids).cuda()
        out = torch.empty((wl.n, wl.out_elems), device="cuda")
        ids[9] = 60
        mt.mt_infer(x, ids, wl.n, out)
        ops.attention(1)
        assert mt.mt_get_async_status() == (2, 9)                # request 9, not sequence 1
        assert mt.mt_get_async_status() == (0, -1)
    finally:
        mt.mt_shutdown()
