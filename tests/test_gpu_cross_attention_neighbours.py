"""mt_cross_attention: the bits of a row depend on its own query and states, and on the sizes of the call (which cut the work into shares), not on what other rows
or sequences hold."""
import pytest
import torch

from lm_util import init
from paper_1901_06887_b200 import binding as mt
from test_gpu_cross_attention import i32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,states,hq,hk", [([1, 1, 1], [1500, 900, 40], 8, 2), ([1] * 9, [130] * 9, 6, 2), ([200, 60, 5], [700, 300, 129], 4, 4),
                                               ([300] * 12, [100 + 77 * i for i in range(12)], 32, 8), ([3, 0, 260], [0, 128, 5000], 5, 1)])
def test_what_the_neighbours_hold(lens, states, hq, hk, dim):
    init()
    q, k, v, offsets, ranges = make(lens, states, hq, hk, dim)
    first, other = torch.empty_like(q), torch.empty_like(q)
    mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), first)
    g = torch.Generator(device="cuda").manual_seed(9)
    noise = lambda t: (20 * torch.randn(t.shape, generator=g, device="cuda")).to(t.dtype)
    for s in {0, len(lens) // 2, len(lens) - 1}:
        if lens[s] == 0:
            continue
        lo, hi = ranges[s]
        for row in {offsets[s], offsets[s] + lens[s] // 2, offsets[s + 1] - 1}:
            q2, k2, v2 = noise(q), noise(k), noise(v)
            q2[(row + 1) % len(q)] = float("nan")
            q2[row], k2[lo:hi], v2[lo:hi] = q[row], k[lo:hi], v[lo:hi]
            mt.mt_cross_attention(q2, k2, v2, i32(offsets), i32(ranges), other)
            assert torch.equal(other[row].view(torch.int16), first[row].view(torch.int16)), (s, row)
    # and from run to run
    mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), other)
    assert torch.equal(other.view(torch.int16), first.view(torch.int16))
    assert mt.mt_get_async_status() == (0, -1)
