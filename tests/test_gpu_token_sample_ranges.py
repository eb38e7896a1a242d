"""mt_token_sample at the ends of what its arguments may be."""
import numpy as np
import pytest
import torch

from lm_util import to_np
from more_lm_util import sample_bound
from paper_1901_06887_b200 import binding as mt
from test_gpu_token_sample import arrays, check, draw, init, random_logits

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [1, 2, 5, 1000, 40000])
@pytest.mark.parametrize("p", [-3.0, -1e4, -3e38, -float("inf")])
def test_top_p_far_below_zero(p, v, dtype):
    """Any share below zero is reached by the first entry; with a limit on the count, too."""
    n = 9
    x, u, _ = random_logits(n, v, dtype, 11)
    first = to_np(x).argmax(1)
    assert (check(x, u, **arrays(n, dict(top_p=p))) == first).all()
    assert (check(x, u, **arrays(n, dict(top_p=p, top_k=3, temperature=0.7))) == first).all()
    assert mt.mt_get_async_status() == (0, -1)
