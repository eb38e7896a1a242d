"""What the binding's calls of the language-model operators refuse before the library sees it: tensors of another rank, on
another device, sizes and numbers that the C interface cannot take.  Always MtError with MT_ERR_INVALID_ARG."""
import pytest
import torch

from lm_util import code_of, init
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


class Elsewhere:
    """A tensor that says it lies on the next GPU (its memory lies on this one)."""

    def __init__(self, t):
        self.t = t

    def get_device(self):
        return self.t.get_device() + 1

    @property
    def device(self):
        return torch.device("cuda", self.get_device())

    def __getattr__(self, name):
        return getattr(self.t, name)


class Huge(Elsewhere):
    """A tensor that says it has 2^32 rows more than it has."""

    def get_device(self):
        return self.t.get_device()

    @property
    def shape(self):
        return torch.Size([self.t.shape[0] + (1 << 32), *self.t.shape[1:]])

    def numel(self):
        return self.t.numel() // self.t.shape[0] * self.shape[0]


def calls():
    """name -> (function, arguments that it takes, by position)."""
    init()
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")
    cache = mt.KvCache.empty(2, 16, 2, 64)
    bank = mt.QuantBank(z(2, 8, 32, dtype=torch.uint8), z(2, 8, 1))
    i32 = torch.int32
    return {
        "prompt": (mt.mt_prompt_attention, [z(3, 2, 64), z(3, 2, 64), z(3, 2, 64), torch.tensor([0, 3], dtype=i32, device="cuda"), z(3, 2, 64)]),
        "append": (mt.mt_kv_append, [cache, z(3, 2, 64), z(3, 2, 64), torch.arange(3, device="cuda")]),
        "read": (mt.mt_kv_read, [cache, torch.arange(3, device="cuda"), z(3, 2, 64), z(3, 2, 64)]),
        "attention": (mt.mt_kv_attention, [cache, z(3, 2, 64), z(3, 1, dtype=i32), z(3, dtype=i32), z(3, 2, 64)]),
        "cache": (mt.KvCache, [z(2, 2, 16, 32, dtype=torch.uint8), z(2, 2, 16, 2), z(2, 2, 16, 32, dtype=torch.uint8), z(2, 2, 16, 2)]),
        "pack": (mt.mt_quant_pack, [z(2, 8, 32, dtype=torch.uint8), z(2, 8, 1), z(2, 16 * 32 + 32, dtype=torch.uint8)]),
        "bank": (mt.QuantBank, [z(2, 8, 32, dtype=torch.uint8), z(2, 8, 1), z(2, 8, dtype=torch.float32)]),
        "linear": (mt.mt_quant_linear, [z(3, 64), z(3, dtype=i32), bank, z(3, 8)]),
        "logprobs": (mt.mt_token_logprobs, [z(3, 50), z(3, dtype=i32), z(3, dtype=torch.float32), z(3, dtype=torch.float32), z(3, 2, dtype=i32),
                                            z(3, 2, dtype=torch.float32)]),
    }


NAMES = ["prompt", "append", "read", "attention", "cache", "pack", "bank", "linear", "logprobs"]


@pytest.mark.parametrize("name", NAMES)
def test_rank_and_place(name):
    f, args = calls()[name]
    f(*args)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor):
            continue
        ranks = (t[0],) if name == "pack" and i == 2 else (t[None], t[0])       # (packed weights: any shape that is large enough)
        for other in (*ranks, t.cpu(), Elsewhere(t)):
            assert code_of(f, *args[:i], other, *args[i + 1:]) == 1, (i, type(other), other.shape)
    assert mt.mt_get_async_status() == (0, -1)


@pytest.mark.parametrize("name", ["prompt", "append", "read", "attention", "linear", "logprobs"])
def test_sizes_beyond_32_bits(name):
    """Never cut to their low 32 bits."""
    f, args = calls()[name]
    huge = [Huge(t) if isinstance(t, torch.Tensor) and t.dim() and t.shape[0] == 3 else t for t in args]
    assert code_of(f, *huge) == 1


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf"), 1e39])
@pytest.mark.parametrize("name", ["prompt", "attention"])
def test_scales_that_are_no_numbers(name, scale):
    f, args = calls()[name]
    assert code_of(f, *args, scale=scale) == 1
    f(*args, scale=-3e38)


def test_a_head_dimension_of_zero():
    for name in ("prompt", "append", "read", "attention"):
        f, args = calls()[name]
        args = [t[..., :0] if isinstance(t, torch.Tensor) and t.dim() == 3 else t for t in args]
        assert code_of(f, *args) in (1, 4)
