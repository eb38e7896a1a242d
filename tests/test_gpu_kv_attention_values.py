"""mt_kv_attention where the tokens of a tile differ: value rows of very different size against weights that differ too, and
queries with one element far above the rest.  Held to the same bound as all other decode tests."""
import math

import numpy as np
import pytest
import torch

from lm_util import attention_bound, decode_reference, init, random_cache, to_np
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def check(cache, q, table, n, scale):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    mt.mt_kv_attention(cache, q, torch.tensor([table], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"),
                       out, scale=scale)
    assert mt.mt_get_async_status() == (0, -1)
    o, a = decode_reference(cache, q, [table], [n], scale)
    err = np.abs(to_np(out) - o)
    assert (err <= attention_bound(o, a)).all(), float(np.max(err / attention_bound(o, a)))


def make(n, dim, group, seed):
    """One sequence of n tokens in pages of 32, two key/value heads; queries of positive elements, so that a key row that is
    one number times a bias gets a score of that sign."""
    init()
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = -(-n // 32)
    cache = random_cache(pages, 32, 2, dim, g)
    q = torch.randn((1, 2 * group, dim), generator=g, device="cuda").abs().to(torch.bfloat16)
    return cache, q, list(range(pages)), g


def set_weight(cache, q, token, log_odds, n, scale):
    """Gives `token` a constant key row, for which its weight is about e^log_odds times that of all others together."""
    group = q.shape[1] // cache.heads
    kc, kp = cache.tensors[:2]
    codes = torch.stack([kc & 15, kc >> 4], -1).flatten(-2).double()
    k = codes * kp[..., :1].double() + kp[..., 1:].double()
    for h in range(cache.heads):
        rows = k[:, h].reshape(-1, k.shape[-1])[:n]
        rows = rows[[i for i in range(n) if i != token]]
        qs = q[0, h * group:(h + 1) * group].double()
        lse = torch.logsumexp(rows @ qs.T * scale, 0).mean()
        bias = (lse + log_odds) / (qs.sum(-1).mean() * scale)
        kp[token // 32, h, token % 32] = torch.stack([torch.zeros_like(bias), bias]).to(torch.bfloat16)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 16])
@pytest.mark.parametrize("n", [20, 64, 2048])
@pytest.mark.parametrize("smaller", [20.0, 100.0, 1e4, math.inf])
def test_a_heavy_token_of_small_values(dim, group, n, smaller):
    """What trained models do at their first token: nearly all of the weight, hardly any value."""
    scale = dim ** -0.5
    cache, q, table, _ = make(n, dim, group, seed=n + group)
    cache.tensors[3][0, :, 0] /= smaller
    set_weight(cache, q, 0, 5.0, n, scale)
    check(cache, q, table, n, scale)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 16])
@pytest.mark.parametrize("larger", [1e3, 1e5, 1e20])
@pytest.mark.parametrize("at", [0, 40])
def test_a_large_value_row_without_weight(dim, group, larger, at):
    scale, n = dim ** -0.5, 64
    cache, q, table, _ = make(n, dim, group, seed=group)
    cache.tensors[3][at // 32, :, at % 32] *= larger
    set_weight(cache, q, at, -110.0, n, scale)
    check(cache, q, table, n, scale)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8, 12])
def test_value_rows_of_all_sizes(dim, group):
    """Sizes over five decades inside every tile, under weights over several decades."""
    n = 300
    cache, q, table, g = make(n, dim, group, seed=group)
    vp = cache.tensors[3]
    vp.copy_((vp.float() * 10.0 ** (5 * torch.rand(vp.shape[:-1], generator=g, device="cuda")[..., None] - 3)).to(torch.bfloat16))
    q = torch.randn(q.shape, generator=g, device="cuda").to(torch.bfloat16)
    check(cache, q, table, n, dim ** -0.5)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_appended_rows_of_mixed_size(dim, page):
    """Through the cache's own rounding: rows of keys and values over four decades, written and then attended to."""
    init()
    g = torch.Generator(device="cuda").manual_seed(dim)
    n, heads, group = 333, 2, 4
    size = lambda lo: 10.0 ** (4 * torch.rand((n, heads, 1), generator=g, device="cuda") + lo)
    k = (torch.randn((n, heads, dim), generator=g, device="cuda") * size(-4)).to(torch.bfloat16)
    v = (torch.randn((n, heads, dim), generator=g, device="cuda") * size(-2)).to(torch.bfloat16)
    v[5] = 0.25                                                  # a constant row: scale zero
    k[5] = 1.0
    pages = -(-n // page)
    cache = mt.KvCache.empty(pages, page, heads, dim)
    order = torch.randperm(pages, generator=g, device="cuda")
    at = torch.arange(n, device="cuda")
    mt.mt_kv_append(cache, k, v, order[at // page] * page + at % page)
    q = torch.randn((1, heads * group, dim), generator=g, device="cuda").to(torch.bfloat16)
    q[0, ::2] = q[0, ::2].abs()                                  # these give the constant row most of the weight
    check(cache, q, order.tolist(), n, 2 * dim ** -0.5)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 16])
@pytest.mark.parametrize("top", [16.0, 64.0, 128.0])
def test_a_query_with_one_large_element(dim, group, top):
    """The other elements are alike, so what their rounding takes off adds up over the channels.  The large one meets keys of
    zero.  Half of the keys have codes of ordinary size, the other half hardly any; values tell the two apart."""
    init()
    g = torch.Generator(device="cuda").manual_seed(group)
    n = 64
    cache = random_cache(2, 32, 1, dim, g)
    kc, kp, vc, vp = cache.tensors
    kp[..., 0], kp[..., 1] = 0.25, -1.75
    kp[:, :, ::2] = 0.0
    kc[..., 0] = (kc[..., 0] & 0xf0) | 7                         # channel 0: 7 * 0.25 - 1.75 = 0
    vp[..., 0], vp[..., 1] = 0.0, 1.0
    vp[:, :, ::2, 1] = -1.0
    q = torch.empty((1, group, dim), dtype=torch.bfloat16, device="cuda")
    q[:] = torch.linspace(0.25, 0.75, group, device="cuda")[None, :, None] + 0.0068
    q[:, :, 0] = top
    check(cache, q, [0, 1], n, dim ** -0.5)
