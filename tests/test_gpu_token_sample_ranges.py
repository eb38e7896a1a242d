"""mt_token_sample at the ends of what its arguments may be."""
from fractions import Fraction

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


LARGE = [65536, 131071, 131072, 152064, 262144, 262145, 300000, 1 << 20]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", LARGE)
@pytest.mark.parametrize("n", [1, 5, 300])
def test_equal_logits_of_large_vocabularies(n, v, dtype):
    """Every token weighs as much as the likeliest: the row's mass is the largest there is.  Weights and sums of them are exact, so are the tokens."""
    init()
    x = torch.full((1, v), 1.25, dtype=dtype, device="cuda").expand(n, v)
    u = (torch.arange(n, device="cuda") + 0.75) / n
    for p in (1.0, 0.5, 0.777, 0.99):
        share = Fraction(float(np.float32(p)))
        kept = -(-share.numerator * v // share.denominator)
        ids, logprobs = draw(x, u, **arrays(n, dict(top_p=p)))
        assert ids.tolist() == [int(Fraction(w) * kept) for w in u.tolist()], p
        assert np.abs(logprobs + np.log(kept)).max() <= sample_bound(np.log(kept)), p


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", LARGE)
def test_flat_rows_of_large_vocabularies(v, dtype):
    """A high temperature: masses near the largest, weights of all sizes.  (The sum is off by half a unit a weight, 2^-43 of a weight of most: far less than the bound.)"""
    n = 3
    x, u, _ = random_logits(n, v, dtype, v)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=v // 2), dict(top_k=v // 3, top_p=0.6, min_p=0.3)):
        check(x, u, **arrays(n, dict(temperature=10.0, **kw)))


@pytest.mark.parametrize("v", [262144, 300000])
def test_rows_of_large_vocabularies_do_not_depend_on_the_others(v):
    """Held in parts, or read twice: the same tokens."""
    init()
    n = 160
    x, u, g = random_logits(n, v, BF16, 5)
    kw = arrays(n, dict(temperature=6.0))
    kw["top_p"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.6, torch.rand(n, generator=g, device="cuda"), 1.0)
    ids, logprobs = draw(x, u, **kw)
    for i in range(0, n, 37):
        some = draw(x[i:i + 3], u[i:i + 3].contiguous(), **{k: w[i:i + 3].contiguous() for k, w in kw.items()})
        assert (ids[i:i + 3] == some[0]).all() and (logprobs[i:i + 3] == some[1]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [3, 700, 40000])
@pytest.mark.parametrize("t", [1e35, 1e36, 5e37, 1e38, 3.4e38])
def test_logits_further_apart_than_the_largest_number(t, v, dtype):
    """Temperatures at which the lowest numbers weigh something beside the largest; minus infinity never does."""
    n = 8
    _, u, g = random_logits(n, v, F32, v)
    x = (3.38e38 * (2 * torch.rand((n, v), generator=g, device="cuda") - 1)).to(dtype)
    x[:, 0], x[:, -1] = torch.finfo(dtype).max, torch.finfo(dtype).min
    x[1::2, 1] = -float("inf")
    x[3, 2:] = -float("inf")
    for kw in (dict(), dict(top_k=max(2, v // 3)), dict(top_p=0.6), dict(min_p=0.2), dict(top_k=max(2, v // 2), top_p=0.9, min_p=0.01)):
        check(x, u, **arrays(n, dict(temperature=t, **kw)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [7, 3000, 90000])
def test_minus_zero(v, dtype):
    """The same as zero, in every argument that may be zero."""
    init()
    x, u, _ = random_logits(6, v, dtype, 13)
    u.zero_()
    for kw in (dict(), dict(top_p=0.8), dict(top_k=5, min_p=0.01)):
        plus, minus = draw(x, u, **arrays(6, kw)), draw(x, -u, **arrays(6, kw))
        assert (plus[0] == minus[0]).all() and (plus[1] == minus[1]).all() and (plus[0] >= 0).all()
        check(x, -u, **arrays(6, kw))
    u += 0.4
    for name in ("temperature", "top_p", "min_p"):
        plus, minus = draw(x, u, **arrays(6, {name: 0.0})), draw(x, u, **arrays(6, {name: -0.0}))
        assert (plus[0] == minus[0]).all() and (plus[1] == minus[1]).all()
    assert mt.mt_get_async_status() == (0, -1)
