"""A bank packed on a stream of its own."""
import pytest
import torch

from lm_util import init
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def stream_of(t):
    """The stream that torch's allocator took t's memory for."""
    at = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not torch's memory")


def test_the_packed_weights_belong_to_the_stream_that_packs_them():
    """Memory of the current stream may still be in use there when another stream starts to pack."""
    init()
    g = torch.Generator(device="cuda").manual_seed(0)
    codes = torch.randint(0, 256, (2, 1024, 512), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.ones((2, 1024, 16), dtype=torch.bfloat16, device="cuda")
    want = mt.QuantBank(codes, scales)
    assert stream_of(want.packed) == torch.cuda.current_stream().cuda_stream
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):                      # an object or a handle
        bank = mt.QuantBank(codes, scales, stream=stream)
        torch.cuda.synchronize()
        assert stream_of(bank.packed) == side.cuda_stream
        assert torch.equal(bank.packed, want.packed)
