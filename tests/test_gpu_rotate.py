"""mt_rotate against 64 bits: layouts, axes, partial rotation, far positions, strides, in place, its inverse as its gradient."""
import numpy as np
import pytest
import torch

from lm_util import init, to_np
from more_lm_util import rotate_bound, rotate_reference
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def frequencies(half, base=10000.0):
    return (base ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()


def positions(n, axes, gen, far=4000):
    return torch.randint(0, far, (n, axes), generator=gen, device="cuda", dtype=torch.int32)


def check(x, pos, f, sections=None, neighbours=False, inverse=False, out=None):
    init()
    cut = [len(f)] if sections is None else sections
    want, size = rotate_reference(x, pos, f, cut, neighbours, inverse)
    out = torch.full(x.shape, 77.0, dtype=x.dtype, device="cuda") if out is None else out
    mt.mt_rotate(x, pos, f, out, sections=sections, neighbours=neighbours, inverse=inverse)
    turns = float(pos.double().abs().max() * f.double().abs().max()) / 6.28 + 1 if pos.numel() else 1
    err = np.abs(to_np(out) - want)
    assert (err <= rotate_bound(want, size, x.dtype is BF16, turns)).all(), err.max()
    return out


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,heads,dim,rotary,cut", [
    (1, 1, 16, 16, None), (3, 2, 64, 64, None), (65, 40, 128, 128, None), (7, 5, 128, 64, None), (130, 3, 80, 80, [10, 14, 16]), (9, 7, 256, 256, [64, 64]),
    (33, 1, 96, 32, [16, 0]), (4, 6, 512, 512, [1, 2, 3, 250]), (1000, 9, 64, 48, [8, 8, 8]), (17, 3, 24, 16, [0, 8]), (2, 300, 128, 128, [16, 24, 24])])
def test_shapes(n, heads, dim, rotary, cut, dtype, neighbours):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn((n, heads, dim), generator=g, device="cuda").to(dtype)
    pos = positions(n, len(cut) if cut else 1, g)
    check(x, pos, frequencies(rotary // 2), cut, neighbours)
    check(x, pos, frequencies(rotary // 2), cut, neighbours, inverse=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_axis_may_be_flat(dtype):
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((20, 4, 64), generator=g, device="cuda").to(dtype)
    pos = positions(20, 1, g)
    a, b = check(x, pos, frequencies(32)), check(x, pos[:, 0].contiguous(), frequencies(32))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_and_negative_positions(dtype):
    """A million steps and the largest positions there are, both ways."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((8, 3, 128), generator=g, device="cuda").to(dtype)
    pos = torch.tensor([0, 1, -1, 10 ** 6, -10 ** 6, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32, device="cuda")
    check(x, pos, frequencies(64))
    check(x, pos, frequencies(64, 1e6), neighbours=True)
    check(x[:5], pos[:5].contiguous(), 50.0 * frequencies(64))  # more than a turn a step


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rotary", [64, 32])
def test_slices_and_in_place(dtype, rotary):
    """Queries and keys inside one projection's output, turned where they lie; what lies around them stays."""
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn((50, 11, 72), generator=g, device="cuda").to(dtype)
    before, pos, f = qkv.clone(), positions(50, 2, g), frequencies(rotary // 2)
    cut = [rotary // 4, rotary // 4]
    x = qkv[:, 2:8, 8:]
    want = check(x, pos, f, cut)
    wide = torch.full((50, 9, 80), 5.0, dtype=dtype, device="cuda")
    check(x, pos, f, cut, out=wide[:, 1:7, 8:72])
    assert (wide[:, 0] == 5).all() and (wide[:, 7:] == 5).all() and (wide[..., :8] == 5).all() and (wide[..., 72:] == 5).all()
    mt.mt_rotate(x, pos, f, x, sections=cut)
    assert torch.equal(x, want)
    rest = qkv.clone()
    rest[:, 2:8, 8:] = before[:, 2:8, 8:]
    assert torch.equal(rest, before)
    heads = torch.randn((6, 30, 64), generator=g, device="cuda").to(dtype).transpose(0, 1)            # heads outside, tokens inside
    check(heads, positions(30, 1, g), frequencies(32))


def test_shared_rows():
    """A stride of zero between tokens: one row turned to many positions."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((1, 4, 64), generator=g, device="cuda").to(BF16).expand(30, 4, 64)
    check(x, positions(30, 1, g), frequencies(32))


def test_values_that_are_no_numbers_stay_in_their_pair():
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((4, 3, 64), generator=g, device="cuda").to(BF16)
    pos, f = positions(4, 1, g), frequencies(32)
    clean = check(x, pos, f)
    x[1, 2, 5], x[2, 0, 40] = float("nan"), float("inf")
    out = torch.empty_like(x)
    mt.mt_rotate(x, pos, f, out)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 2, [5, 37]] = bad[2, 0, [8, 40]] = True
    assert torch.equal(out[~bad], clean[~bad]) and not torch.isfinite(out[bad]).any()


@pytest.mark.parametrize("neighbours", [False, True])
def test_the_inverse_is_the_gradient(neighbours):
    """Against the formula's gradient by torch and against differences, in fp32."""
    init()
    g = torch.Generator(device="cuda").manual_seed(5)
    x, d = (torch.randn((6, 2, 32), generator=g, device="cuda") for _ in range(2))
    pos, f = positions(6, 2, g, 50), frequencies(16)
    cut = [9, 7]
    got = torch.empty_like(d)
    mt.mt_rotate(d, pos, f, got, sections=cut, neighbours=neighbours, inverse=True)
    axis = torch.repeat_interleave(torch.arange(2), torch.tensor(cut)).cuda()
    angle = (pos.double()[:, axis] * f.double())[:, None]
    y = x.double().requires_grad_()
    a, b = (y[..., 0::2], y[..., 1::2]) if neighbours else (y[..., :16], y[..., 16:])
    turned = (a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos())
    z = torch.stack(turned, -1).flatten(-2) if neighbours else torch.cat(turned, -1)
    (z * d.double()).sum().backward()
    assert (got.double() - y.grad).abs().max() <= 16 * 2.0 ** -24 * 8
    # differences: the turning is linear, so a step of one is exact up to rounding
    out0, out1, e = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(x)
    mt.mt_rotate(x, pos, f, out0, sections=cut, neighbours=neighbours)
    for t, h, c in ((0, 0, 0), (3, 1, 17), (5, 0, 31)):
        e.zero_()
        e[t, h, c] = 1.0
        mt.mt_rotate(x + e, pos, f, out1, sections=cut, neighbours=neighbours)
        slope = ((out1.double() - out0.double()) * d.double()).sum().item()
        assert abs(slope - got[t, h, c].item()) <= 64 * 2.0 ** -24 * 8


def test_captured_and_on_another_stream():
    init()
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((40, 4, 64), generator=g, device="cuda").to(BF16)
    pos, f, out = positions(40, 1, g), frequencies(32), torch.empty_like(x)
    want = check(x, pos, f)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.mt_rotate(x, pos, f, out, stream=torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    mt.mt_rotate(x, pos, f, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    mt.mt_rotate(x[:0], pos[:0], f, out[:0])
