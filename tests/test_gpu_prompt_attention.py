"""mt_prompt_attention against a 64-bit implementation: lengths from one token, packed sequences, grouped heads, strides,
masked infinities, refusals."""
import numpy as np
import pytest
import torch

from lm_util import attention_bound, code_of, init, prompt_reference
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def make(lens, hq, hkv, d, seed=0, size=1.0):
    init()
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(lens)
    qkv = (torch.randn((n, hq + 2 * hkv, d), generator=g, device="cuda") * size).to(torch.bfloat16)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], off


def check(q, k, v, off, scale=None, **kw):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    mt.mt_prompt_attention(q, k, v, torch.from_numpy(off).cuda(), out, scale=scale, **kw)
    torch.cuda.synchronize()
    assert mt.mt_get_async_status() == (0, -1)
    o, a = prompt_reference(q, k, v, off.tolist(), q.shape[2] ** -0.5 if scale is None else scale)
    got = out.double().cpu().numpy()
    inside = ~np.isnan(o)
    assert (got[~inside] == 7.0).all()                 # rows of no sequence are not written
    err = np.abs(got - o)[inside]
    assert (err <= attention_bound(o, a)[inside]).all(), float(np.max(err / attention_bound(o, a)[inside]))
    return out


@pytest.mark.parametrize("lens", [[1], [2], [17], [127], [128], [129], [255, 1], [256], [257], [1, 1, 1, 1], [300, 0, 5, 64],
                                  [0, 0, 130], [513], [40, 700, 3, 90]])
@pytest.mark.parametrize("heads", [(2, 1, 64), (4, 4, 64), (8, 1, 128), (2, 2, 128)])
def test_lengths(lens, heads):
    check(*make(lens, *heads, seed=len(lens)))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (6, 2), (7, 1), (12, 3), (16, 1), (32, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_head_groups(hq, hkv, d):
    check(*make([150, 33], hq, hkv, d, seed=hq))


def test_many_short_sequences():
    rng = np.random.default_rng(3)
    check(*make(rng.integers(0, 20, 700).tolist(), 2, 1, 64))


def test_long_sequence_and_sharp_scores():
    check(*make([2100], 2, 1, 128, size=1.0))
    check(*make([1500], 2, 1, 64, size=3.0), scale=0.05)


def test_scale_zero_and_negative():
    q, k, v, off = make([200, 9], 2, 1, 64)
    check(q, k, v, off, scale=0.0)
    check(q, k, v, off, scale=-0.1)


def test_rows_outside_the_sequences_are_left():
    q, k, v, _ = make([300], 2, 1, 64)
    check(q, k, v, np.array([10, 150, 290], np.int32))


def test_strides():
    init()
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((4, 190, 136), generator=g, device="cuda").to(torch.bfloat16)[:, :, 8:].transpose(0, 1)   # heads outermost
    k = torch.randn((190, 2, 128), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((190, 6, 128), generator=g, device="cuda").to(torch.bfloat16)[:, ::3]
    check(q, k, v, np.array([0, 61, 190], np.int32))


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan"), 3.38e38, -3.38e38])
@pytest.mark.parametrize("d", [64, 128])
def test_masked_values_never_show(what, d):
    """Infinities, NaN and the type's extremes in k and v of later tokens and of other sequences."""
    lens = [70, 200, 90]
    q, k, v, off = make(lens, 4, 2, d, seed=5)
    clean = check(q, k, v, off)
    k2, v2 = k.clone(), v.clone()
    k2[off[1] + 150:off[2]] = what                     # the second sequence goes wrong at its 150th token
    v2[off[1] + 150:off[2]] = what
    k2[off[2]:], v2[off[2]:] = what, what              # the third altogether
    out = torch.empty_like(clean)
    mt.mt_prompt_attention(q, k2, v2, torch.from_numpy(off).cuda(), out)
    torch.cuda.synchronize()
    assert torch.equal(out[:off[1] + 150], clean[:off[1] + 150])
    if not abs(what) < 1e39:                           # what may see them is not finite
        assert not torch.isfinite(out[off[2]:]).any()


def test_single_bad_value_in_the_middle():
    q, k, v, off = make([260], 2, 1, 128, seed=6)
    clean = check(q, k, v, off)
    v2 = v.clone()
    v2[131, 0, 5] = float("nan")
    out = torch.empty_like(clean)
    mt.mt_prompt_attention(q, k, v2, torch.from_numpy(off).cuda(), out)
    torch.cuda.synchronize()
    assert torch.equal(out[:131], clean[:131])
    assert torch.isnan(out[131:, :, 5]).all()
    keep = [i for i in range(128) if i != 5]
    assert torch.equal(out[131:, :, keep], clean[131:, :, keep])


def test_broken_offsets_are_refused_on_the_device():
    q, k, v, _ = make([100], 2, 1, 64)
    for off, bad in (([0, 40, 30, 100], 1), ([0, 40, 101], 1), ([-1, 40], 0)):
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        mt.mt_prompt_attention(q, k, v, torch.tensor(off, dtype=torch.int32, device="cuda"), out)
        assert mt.mt_get_async_status() == (1, bad)
        if bad == 1:                                   # the sequence before it is complete (up to where the first case's third overlaps it)
            o, a = prompt_reference(q, k, v, [0, 40], 0.125)
            assert (np.abs(out.double().cpu().numpy() - o)[:30] <= attention_bound(o, a)[:30]).all()
    assert mt.mt_get_async_status() == (0, -1)


def test_refusals():
    q, k, v, off = make([16], 4, 2, 64)
    off = torch.from_numpy(off).cuda()
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    f = mt.mt_prompt_attention
    assert code_of(f, q.float(), k, v, off, out) == 1
    assert code_of(f, q, k, v, off.long(), out) == 1
    assert code_of(f, q, k[:, :, :32], v, off, out) == 1
    assert code_of(f, q, k, v, off, out[:8]) == 1
    assert code_of(f, q[:, :3], k, v, off, out[:, :3].contiguous()) == 4          # 3 heads over 2
    x = torch.zeros((16, 2, 96), dtype=torch.bfloat16, device="cuda")
    assert code_of(f, x, x, x, off, x.clone()) == 4                               # head_dim 96
    x = torch.zeros((16, 2, 65), dtype=torch.bfloat16, device="cuda")[:, :, :64]  # head stride 65
    assert code_of(f, x, x, x, off, x.contiguous()) == 4
    x = torch.zeros(16 * 128 + 8, dtype=torch.bfloat16, device="cuda")[1:16 * 128 + 1].view(16, 2, 64)   # 2 bytes off
    assert code_of(f, x, x, x, off, x.clone()) == 1
    e = q[:0]
    f(e, k[:0], v[:0], off, out[:0])                                              # no tokens: nothing to do
    f(q, k, v, off[:1], out)                                                      # no sequences
    assert mt.mt_get_async_status() == (0, -1)


def test_other_stream_and_graph():
    q, k, v, off = make([90, 222], 4, 2, 128, seed=9)
    want = check(q, k, v, off)
    s = torch.cuda.Stream()
    out = torch.zeros_like(want)
    d_off = torch.from_numpy(off).cuda()
    s.wait_stream(torch.cuda.current_stream())
    mt.mt_prompt_attention(q, k, v, d_off, out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.mt_prompt_attention(q, k, v, d_off, out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_scores_that_rise_along_the_sequence():
    """Each 128 keys lie far above all before them, by less and by more than what the running reference allows, and fall again."""
    for step in (5.0, 40.0, 400.0, 3000.0):
        q, k, v, off = make([700], 2, 1, 64, seed=11)
        q, k = q.clone(), 0.1 * k
        q[..., 0] = 1.0
        level = torch.tensor([0, 1, 2, 4, 3, 5], device="cuda")[torch.arange(700, device="cuda") // 128]
        k[:, 0, 0] = (level * step).to(torch.bfloat16)
        k[300, 0, 0] = k[300, 0, 0] + torch.tensor(2 * step, device="cuda").to(torch.bfloat16)     # one key inside a block, in its first half
        k[480, 0, 0] = k[480, 0, 0] + torch.tensor(3 * step, device="cuda").to(torch.bfloat16)     # and one in a second half
        check(q, k, v, off, scale=0.5)


def test_first_block_without_weight():
    """Scores of minus infinity in all of the first 128 keys; the rest decides, however low it lies."""
    q, k, v, off = make([400], 1, 1, 64, seed=12)
    q, k = q.clone(), k.clone()
    q[..., 0] = 1.0
    k[:128, 0, 0] = float("-inf")
    k[128:, 0, 0] = -1000.0
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    mt.mt_prompt_attention(q, k, v, torch.from_numpy(off).cuda(), out)
    torch.cuda.synchronize()
    o, a = prompt_reference(q[128:], k[128:], v[128:], [0, 272], 0.125)       # the first 128 keys weigh nothing
    assert (np.abs(out[128:].double().cpu().numpy() - o) <= attention_bound(o, a)).all()
    assert torch.isnan(out[:128]).all()
