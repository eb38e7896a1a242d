"""mt_quant_pack and mt_quant_linear against a 64-bit implementation."""
import numpy as np
import pytest
import torch

from lm_util import code_of, init, linear_bound, linear_reference, to_np
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def make(tenants, k, n, group, seed=0, bias=True):
    init()
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (tenants, n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (0.5 + torch.rand((tenants, n, k // group), generator=g, device="cuda")).to(torch.bfloat16) / 16
    b = torch.randn((tenants, n), generator=g, device="cuda") if bias else None
    return codes, scales, b, g


def check(codes, scales, bias, ids, g, dtype=torch.float32, x=None, y=None):
    k = 2 * codes.shape[2]
    bank = mt.QuantBank(codes, scales, bias)
    if x is None:
        x = torch.randn((len(ids), k), generator=g, device="cuda").to(torch.bfloat16)
    if y is None:
        y = torch.full((len(ids), codes.shape[1]), 7.0, dtype=dtype, device="cuda")
    mt.mt_quant_linear(x, torch.tensor(ids, dtype=torch.int32, device="cuda"), bank, y)
    assert mt.mt_get_async_status() == (0, -1)
    want, a = linear_reference(x, ids, codes, scales, bias)
    err = np.abs(to_np(y) - want)
    bound = linear_bound(want, a, k, y.dtype == torch.bfloat16)
    assert (err <= bound).all(), float(np.max(err / bound))
    return y


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("k", [128, 384, 1024])
@pytest.mark.parametrize("n", [1, 7, 16, 17, 130])
def test_sizes(group, k, n):
    codes, scales, bias, g = make(2, k, n, group, seed=k + n)
    check(codes, scales, bias, [1, 0, 1], g)


@pytest.mark.parametrize("k,group", [(64, 32), (64, 64), (192, 192), (320, 64), (4096, 4096), (8192, 64), (16384, 32)])
def test_inner_sizes(k, group):
    codes, scales, bias, g = make(1, k, 40, group, seed=k, bias=False)
    check(codes, scales, bias, [0], g)
    check(codes, scales, bias, [0] * 9, g)


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 64, 65, 100])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_one_tenant(rows, dtype):
    codes, scales, bias, g = make(3, 256, 70, 64, seed=rows)
    check(codes, scales, bias, [2] * rows, g, dtype)


@pytest.mark.parametrize("rows,tenants", [(24, 8), (64, 64), (200, 3), (300, 40), (600, 2), (5, 1000)])
def test_mixed_batches(rows, tenants):
    codes, scales, bias, g = make(tenants, 128, 33, 64, seed=rows)
    check(codes, scales, bias, np.random.default_rng(rows).integers(0, tenants, rows).tolist(), g)


def test_large_layer():
    codes, scales, bias, g = make(2, 2048, 5000, 64, seed=1)
    check(codes, scales, bias, [0, 1, 1, 0, 1, 0, 0, 0, 0, 0, 0], g, torch.bfloat16)


def test_strides_and_unaligned_outputs():
    codes, scales, bias, g = make(2, 128, 19, 64, seed=2)
    wide = torch.randn((6, 200), generator=g, device="cuda").to(torch.bfloat16)
    for dtype in (torch.bfloat16, torch.float32):
        buf = torch.full((6 * 23 + 1,), 7.0, dtype=dtype, device="cuda")
        y = buf[1:].view(6, 23)[:, :19]
        check(codes, scales, bias, [0, 1, 0, 1, 1, 1], g, x=wide[:, 64:192], y=y)
        assert (buf[1:].view(6, 23)[:, 19:] == 7.0).all() and buf[0] == 7.0


def test_codes_scales_and_inputs_at_their_extremes():
    codes, scales, bias, g = make(1, 128, 16, 64, seed=3, bias=False)
    codes[:, 0] = 0x00                      # every weight -8 scales
    codes[:, 1] = 0xff                      # 7 scales
    codes[:, 2] = 0x88                      # zero
    scales[:, 3] = 0.0
    scales[:, 4] = -1.5
    scales[:, 5] = 1e30
    y = check(codes, scales, bias, [0, 0], g)
    assert (y[:, 2:4] == 0).all()


def test_values_that_are_not_finite_stay_in_their_row():
    codes, scales, bias, g = make(2, 128, 40, 64, seed=4)
    x = torch.randn((5, 128), generator=g, device="cuda").to(torch.bfloat16)
    ids = [0, 1, 0, 0, 1]
    want = check(codes, scales, bias, ids, g, x=x)
    x2 = x.clone()
    x2[2, 100] = float("nan")
    x2[4, 3] = float("inf")
    y = torch.empty_like(want)
    mt.mt_quant_linear(x2, torch.tensor(ids, dtype=torch.int32, device="cuda"), mt.QuantBank(codes, scales, bias), y)
    assert torch.equal(y[[0, 1, 3]], want[[0, 1, 3]])
    assert torch.isnan(y[2]).all() and not torch.isfinite(y[4]).any()


def test_ids_outside_the_bank():
    codes, scales, bias, g = make(3, 128, 40, 64, seed=5)
    x = torch.randn((6, 128), generator=g, device="cuda").to(torch.bfloat16)
    bank = mt.QuantBank(codes, scales, bias)
    good = torch.tensor([0, 1, 2, 2, 1, 0], dtype=torch.int32, device="cuda")
    bad = torch.tensor([0, 3, 2, -1, 1, 0], dtype=torch.int32, device="cuda")
    a, b = (torch.empty((6, 40), device="cuda") for _ in range(2))
    mt.mt_quant_linear(x, good, bank, a)
    mt.mt_quant_linear(x, bad, bank, b)
    assert mt.mt_get_async_status() == (2, 1)
    assert torch.isnan(b[[1, 3]]).all() and torch.equal(a[[0, 2, 4, 5]], b[[0, 2, 4, 5]])
    bad.fill_(7)
    mt.mt_quant_linear(x, bad, bank, b)
    assert mt.mt_get_async_status() == (2, 0) and torch.isnan(b).all()
    many = torch.zeros(400, dtype=torch.int32, device="cuda")
    many[300] = 9
    y = torch.empty((400, 40), device="cuda")
    mt.mt_quant_linear(x[:1].expand(400, 128).contiguous(), many, bank, y)
    assert mt.mt_get_async_status() == (2, 300) and torch.isnan(y[300]).all() and int(torch.isnan(y).any(1).sum()) == 1


def test_a_row_does_not_depend_on_its_batch():
    codes, scales, bias, g = make(4, 512, 50, 64, seed=6)
    x = torch.randn((20, 512), generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.arange(20, device="cuda", dtype=torch.int32) % 4
    bank = mt.QuantBank(codes, scales, bias)
    y, one = torch.empty((20, 50), device="cuda"), torch.empty((1, 50), device="cuda")
    mt.mt_quant_linear(x, ids, bank, y)
    for i in (0, 7, 19):
        mt.mt_quant_linear(x[i:i + 1], ids[i:i + 1], bank, one)
        assert torch.equal(one[0], y[i])


def test_refusals():
    codes, scales, bias, g = make(2, 128, 20, 64)
    bank = mt.QuantBank(codes, scales, bias)
    x = torch.zeros((3, 128), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    y = torch.empty((3, 20), device="cuda")
    f = mt.mt_quant_linear
    assert code_of(f, x.float(), ids, bank, y) == 1
    assert code_of(f, x, ids.long(), bank, y) == 1
    assert code_of(f, x[:, :64], ids, bank, y) == 1
    assert code_of(f, x, ids, bank, y[:, :19]) == 1
    assert code_of(f, x, ids, bank, y.half()) == 1
    assert code_of(f, torch.zeros((3, 132), dtype=torch.bfloat16, device="cuda")[:, :128], ids, bank, y) == 4    # row stride 132
    assert code_of(f, torch.zeros((3, 136), dtype=torch.bfloat16, device="cuda")[:, 1:129], ids, bank, y) == 1   # 2 bytes off
    for k, group, code in ((96, 32, 4), (128, 48, 1), (128, 16, 4), (192, 96, 4)):
        c = torch.zeros((1, 4, k // 2), dtype=torch.uint8, device="cuda")
        s = torch.zeros((1, 4, max(1, k // group)), dtype=torch.bfloat16, device="cuda")
        assert code_of(mt.QuantBank, c, s if k % group == 0 else s[:, :, :1].expand(1, 4, 5)) == code
    assert code_of(mt.mt_quant_packed_bytes, 0, 4, 64) == 1
    assert code_of(mt.mt_quant_pack, codes, scales, torch.empty(16, dtype=torch.uint8, device="cuda")) == 1
    f(x[:0], ids[:0], bank, y[:0])
    assert mt.mt_get_async_status() == (0, -1)


def test_other_stream_and_graph():
    codes, scales, bias, g = make(3, 256, 90, 64, seed=7)
    ids = [0, 2, 2, 1]
    x = torch.randn((4, 256), generator=g, device="cuda").to(torch.bfloat16)
    want = check(codes, scales, bias, ids, g, x=x)
    bank, d_ids, y = mt.QuantBank(codes, scales, bias), torch.tensor(ids, dtype=torch.int32, device="cuda"), torch.empty_like(want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    mt.mt_quant_linear(x, d_ids, bank, y, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.mt_quant_linear(x, d_ids, bank, y)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
