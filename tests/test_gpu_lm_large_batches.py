"""Batches beyond what one table of the kernels holds: more tiles a CTA than are looked up at once, more rows than a launch."""
import numpy as np
import pytest
import torch

from lm_util import attention_bound, init, linear_bound, linear_reference, to_np
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_with_hundreds_of_tiles_a_cta(dim):
    """512 prompts of 1 to 3 tokens, 192 heads: every (prompt, head) is a tile, some 660 for each of 148 CTAs."""
    init()
    g = torch.Generator(device="cuda").manual_seed(dim)
    lens, heads = [1 + i % 3 for i in range(512)], 192
    n = sum(lens)
    qkv = torch.randn((3, n, heads, dim), generator=g, device="cuda").to(torch.bfloat16)
    off = np.concatenate([[0], np.cumsum(lens)])
    out = torch.full((n, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    mt.mt_prompt_attention(*qkv, torch.tensor(off, dtype=torch.int32, device="cuda"), out)
    assert mt.mt_get_async_status() == (0, -1)
    q, k, v = qkv.double()
    at = torch.tensor(off[:-1], device="cuda")[:, None] + torch.arange(3, device="cuda")
    there = torch.arange(3, device="cuda")[None] < torch.tensor(lens, device="cuda")[:, None]
    at = at.clamp_max(n - 1)
    s = torch.einsum("sihd,sjhd->shij", q[at], k[at]) * dim ** -0.5
    s = s.masked_fill(torch.ones((3, 3), dtype=torch.bool, device="cuda").triu(1), float("-inf"))
    p = torch.softmax(s, -1)
    o, a = (torch.einsum("shij,sjhd->sihd", p, x)[there].cpu().numpy() for x in (v[at], v[at].abs()))
    assert (np.abs(to_np(out) - o) <= attention_bound(o, a)).all()


@pytest.mark.parametrize("count,hq,hkv,dim", [(200, 32, 8, 128), (500, 4, 4, 64), (130, 48, 48, 64)])
def test_many_prompts_of_one_tile(count, hq, hkv, dim):
    """Short prompts fill one of the two tiles of a CTA only, for many rounds in a row; a few longer ones come first."""
    init()
    g = torch.Generator(device="cuda").manual_seed(count)
    rng = np.random.default_rng(count)
    lens = rng.integers(1, 30, count)
    lens[:: count // 7] = rng.integers(30, 400, len(lens[:: count // 7]))
    off = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = (torch.randn((off[-1], h, dim), generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    v[off[40]] = float("inf")                                    # the first token of one prompt: its rows alone are not finite
    out = torch.full((off[-1], hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    mt.mt_prompt_attention(q, k, v, torch.tensor(off, dtype=torch.int32, device="cuda"), out)
    assert mt.mt_get_async_status() == (0, -1)
    assert not torch.isfinite(out[off[40]:off[41]]).any()
    v[off[40]] = 0.0
    out[off[40]:off[41]] = 0.0
    for a, b in zip(off[:-1], off[1:]):
        if a == off[40]:
            continue
        s = torch.einsum("ihd,jhd->hij", q[a:b].double(), k[a:b].double().repeat_interleave(hq // hkv, 1)) * dim ** -0.5
        p = torch.softmax(s.masked_fill(torch.ones_like(s[0], dtype=torch.bool).triu(1), float("-inf")), -1)
        vv = v[a:b].double().repeat_interleave(hq // hkv, 1)
        o, size = (torch.einsum("hij,jhd->ihd", p, x) for x in (vv, vv.abs()))
        assert ((out[a:b].double() - o).abs() <= torch.from_numpy(attention_bound(o.cpu().numpy(), size.cpu().numpy())).cuda()).all()


@pytest.mark.parametrize("rows,tenants", [(601, 1), (1025, 7), (3000, 300)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_rows_through_a_layer(rows, tenants, dtype):
    init()
    g = torch.Generator(device="cuda").manual_seed(rows)
    k, n = 256, 50
    codes = torch.randint(0, 256, (tenants, n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = ((0.5 + torch.rand((tenants, n, k // 64), generator=g, device="cuda")) / 16).to(torch.bfloat16)
    bias = torch.randn((tenants, n), generator=g, device="cuda")
    x = torch.randn((rows, k), generator=g, device="cuda").to(torch.bfloat16)
    ids = np.random.default_rng(rows).integers(0, tenants, rows)
    ids.sort()                                                   # prompts one behind the other
    y = torch.full((rows, n), 7.0, dtype=dtype, device="cuda")
    mt.mt_quant_linear(x, torch.tensor(ids, dtype=torch.int32, device="cuda"), mt.QuantBank(codes, scales, bias), y)
    assert mt.mt_get_async_status() == (0, -1)
    want, a = linear_reference(x, ids.tolist(), codes, scales, bias)
    assert (np.abs(to_np(y) - want) <= linear_bound(want, a, k, dtype == torch.bfloat16)).all()
