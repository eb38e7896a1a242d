"""mt_cross_attention at scales near the largest number and near zero."""
import numpy as np
import pytest
import torch

from lm_util import attention_bound, init, to_np
from more_lm_util import cross_reference
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("scale", [2.35e38, -2.35e38, 2.0 ** 100, -(2.0 ** 100), 2.0 ** -90, 0.0])
@pytest.mark.parametrize("dim,lens", [(64, [1, 30]), (128, [1, 30]), (128, [300, 7])])
def test_scales(scale, dim, lens):
    """Queries so small (or large) that the scores are of ordinary size, and queries of zero.  (At the largest scales the former would be no normal numbers.)"""
    init()
    g = torch.Generator(device="cuda").manual_seed(3)
    n, states = sum(lens), [200, 77]
    q = torch.randn((n, 2, dim), generator=g, device="cuda").to(BF16)
    if abs(scale) > 1e38:
        q.zero_()
    elif scale:
        q = (q.float() * 2.0 ** -round(np.log2(abs(scale) * dim ** 0.5))).to(BF16)
    q[::3] = 0
    k, v = (torch.randn((sum(states), 1, dim), generator=g, device="cuda").to(BF16) for _ in range(2))
    offsets, ranges = [0, lens[0], n], [[0, states[0]], [states[0], sum(states)]]
    out = torch.empty_like(q)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), out, scale=scale)
    o, a = cross_reference(q, k, v, offsets, ranges, scale)
    assert (np.abs(to_np(out) - o) <= attention_bound(o, a)).all()
    assert mt.mt_get_async_status() == (0, -1)
