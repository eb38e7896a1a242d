"""mt_cross_attention against 64 bits: lengths from none to long, shared and padded states, heads, strides, pieces that are joined, masked garbage."""
import numpy as np
import pytest
import torch

from lm_util import attention_bound, init, to_np
from more_lm_util import cross_reference
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(lens, states, hq, hk, dim, seed=0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((sum(lens), hq, dim), generator=g, device="cuda").to(BF16)
    kv = torch.randn((sum(states), 2 * hk, dim), generator=g, device="cuda")
    kv[..., 3::37] *= 3
    kv = (kv + shift).to(BF16)
    edges = np.concatenate([[0], np.cumsum(states)])
    return q, kv[:, :hk], kv[:, hk:], [0] + np.cumsum(lens).tolist(), [[int(a), int(b)] for a, b in zip(edges[:-1], edges[1:])]


def check(q, k, v, offsets, ranges, scale=None):
    init()
    out = torch.full(q.shape, 77.0, dtype=BF16, device="cuda")
    mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), out, scale)
    assert mt.mt_get_async_status() == (0, -1)
    o, a = cross_reference(q, k, v, offsets, ranges, q.shape[-1] ** -0.5 if scale is None else scale)
    got, written = to_np(out), ~np.isnan(o)
    assert (got[~written] == 77).all()
    err = np.abs(got - o)[written]
    assert (err <= attention_bound(o, a)[written]).all(), (err / attention_bound(o, a)[written]).max()
    return out


@pytest.mark.parametrize("hq,hk,dim", [(1, 1, 64), (8, 2, 128), (4, 4, 64), (6, 2, 128), (32, 2, 64), (7, 1, 128), (20, 4, 64)])
@pytest.mark.parametrize("lens,states", [([1], [1]), ([1], [1500]), ([3, 1, 70], [129, 128, 127]), ([130, 1, 0, 300], [5, 700, 30, 256]), ([513], [640])])
def test_shapes(lens, states, hq, hk, dim):
    check(*make(lens, states, hq, hk, dim, sum(lens)))


@pytest.mark.parametrize("n", [1, 2, 127, 128, 129, 255, 256, 257, 383, 1025, 20000])
def test_states(n):
    """Ends of blocks of states, one token and a few."""
    check(*make([1], [n], 4, 2, 128, n))
    check(*make([40], [n], 3, 3, 64, n))


@pytest.mark.parametrize("seqs", [1, 2, 5, 64, 150])
@pytest.mark.parametrize("hq,hk,dim", [(8, 2, 128), (5, 5, 64)])
def test_a_token_step(seqs, hq, hk, dim):
    rng = np.random.default_rng(seqs)
    check(*make([1] * seqs, rng.integers(0, 900, seqs).tolist(), hq, hk, dim, seqs))


def test_shared_and_padded_states():
    """Answers that share states, overlapping ranges, rows of a padded batch."""
    q, k, v, offsets, _ = make([1, 1, 9, 40, 3], [1000], 8, 2, 128)
    check(q, k, v, offsets, [[0, 500], [0, 500], [100, 612], [999, 1000], [0, 1000]])


def test_sequences_without_states_give_zeros():
    q, k, v, offsets, _ = make([3, 1, 200], [50], 4, 2, 64)
    out = check(q, k, v, offsets, [[7, 7], [0, 50], [50, 50]])
    assert (out[:3] == 0).all() and (out[4:] == 0).all()
    out = check(q, k[:0], v[:0], offsets, [[0, 0]] * 3)
    assert (out == 0).all()


def test_rows_outside_every_sequence_stay():
    q, k, v, _, _ = make([100], [300], 4, 4, 64)
    check(q, k, v, [5, 20, 20, 90], [[0, 300], [0, 10], [3, 200]])


def test_nothing_else_shows():
    """Infinities and NaN in states of others, and behind the last."""
    q, k, v, offsets, _ = make([2, 150, 1], [700], 8, 4, 128)
    ranges = [[0, 100], [200, 457], [460, 600]]
    want = check(q, k, v, offsets, ranges)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for x in (k, v):
            for lo, hi in ((100, 200), (457, 460), (600, 700)):
                x[lo:hi] = bad
        out = torch.empty_like(q)
        mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), out)
        assert torch.equal(out, want)
    # in a state that is seen, a NaN shows in its sequence and head, and in no other
    v[210, 1, 5] = float("nan")
    mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), out)
    hit = torch.isnan(out)
    assert hit[2:152, 2:4, 5].all() and int(hit.sum()) == 300 and torch.equal(out[~hit], want[~hit])


def test_scores_that_rise_and_that_are_minus_infinity():
    """The running reference has to move, in one piece and between pieces; keys without weight in front."""
    q, k, v, offsets, ranges = make([1, 90], [1300, 1300], 4, 2, 64)
    q = (q.abs() + 0.5).to(BF16)
    k = (k * 0.05 + torch.linspace(-20, 20, 2600, device="cuda")[:, None, None]).to(BF16)
    check(q, k, v, offsets, ranges)
    check(q, (-k.float()).to(BF16), v, offsets, ranges)
    check(q, k, v, offsets, ranges, scale=-0.3)
    check(q, k, v, offsets, ranges, scale=0.0)
    k = torch.full_like(k, 0.01)
    k[:400] = k[1300:1500] = -float("inf")
    got = torch.empty_like(q)
    mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), got)
    o, a = cross_reference(q, k[400:], v[400:], offsets, [[0, 900], [1100, 2200]], 0.125)
    assert (np.abs(to_np(got) - o) <= attention_bound(o, a)).all()


def test_strides():
    g = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn((2, 6, 60, 128), generator=g, device="cuda").to(BF16)[1].transpose(0, 1)[3:43]         # heads outside
    k = torch.randn((4, 500, 136), generator=g, device="cuda").to(BF16).transpose(0, 1)[..., 8:]
    v = torch.randn((500, 2, 256), generator=g, device="cuda").to(BF16)[..., 128:]
    check(q, k[:, 1:3], v, [0, 1, 40], [[10, 400], [0, 500]])


@pytest.mark.parametrize("lens,states,hq,hk", [([2000, 1300], [1800, 200], 8, 8), ([9000], [300], 16, 1), ([300] * 30, [130] * 30, 8, 2), ([1] * 700, [100] * 700, 4, 4)])
def test_many_tile_pairs(lens, states, hq, hk):
    """Shares of whole tile pairs, several a CTA, and more sequences than one launch takes."""
    check(*make(lens, states, hq, hk, 64, len(lens)))


def test_bits_do_not_depend_on_the_neighbours_or_the_run():
    q, k, v, offsets, ranges = make([5, 70, 1], [900, 2000, 333], 8, 2, 128)
    a, b = check(q, k, v, offsets, ranges), check(q, k, v, offsets, ranges)
    assert torch.equal(a, b)


def test_sequences_that_are_left_out():
    q, k, v, _, _ = make([60], [200], 4, 2, 64)
    for offsets, ranges, index in (([0, 20, 10, 60], [[0, 9]] * 3, 1), ([-1, 20, 30, 60], [[0, 9]] * 3, 0), ([0, 20, 30, 61], [[0, 9]] * 3, 2),
                                   ([0, 20, 30, 60], [[0, 9], [5, 4], [0, 9]], 1), ([0, 20, 30, 60], [[0, 9], [0, 201], [-1, 3]], 1),
                                   ([0, 20, 30, 60], [[-1, 9], [0, 9], [0, 9]], 0)):
        init()
        out = torch.full(q.shape, 77.0, dtype=BF16, device="cuda")
        mt.mt_cross_attention(q, k, v, i32(offsets), i32(ranges), out)
        assert mt.mt_get_async_status() == (1, index)
        for s in range(3):
            lo, hi, (a, b) = offsets[s], offsets[s + 1], ranges[s]
            good = 0 <= lo <= hi <= 60 and 0 <= a <= b <= 200
            if good:
                o, size = cross_reference(q, k, v, [0] * s + [lo, hi], [[0, 0]] * s + [[a, b]], 0.125)
                assert (np.abs(to_np(out[lo:hi]) - o[lo:hi]) <= attention_bound(o, size)[lo:hi]).all()
        if index == 0 and offsets[0] == 0:
            assert (out[:20] == 77).all()


def test_captured_on_streams_and_beside_each_other():
    """Pieces lie in scratch: of a stream, or of a graph."""
    init()
    q, k, v, offsets, ranges = make([1, 30, 1], [3000, 500, 1500], 8, 2, 128)
    o, r = i32(offsets), i32(ranges)
    want = check(q, k, v, offsets, ranges)
    q2 = (q.float() * 0.5).to(BF16)
    want2 = check(q2, k, v, offsets, ranges)
    out, out2, out3 = (torch.empty_like(q) for _ in range(3))
    graphs = []
    for x, y in ((q, out), (q2, out2)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            mt.mt_cross_attention(x, k, v, o, r, y, stream=torch.cuda.current_stream())
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(20):
        out.zero_(); out2.zero_(); out3.zero_()
        torch.cuda.synchronize()
        for s, f in zip(streams, (graphs[0].replay, graphs[1].replay, lambda: mt.mt_cross_attention(q, k, v, o, r, out3, stream=streams[2]))):
            with torch.cuda.stream(s):
                f()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want2) and torch.equal(out3, want)
    assert mt.mt_get_async_status() == (0, -1)
