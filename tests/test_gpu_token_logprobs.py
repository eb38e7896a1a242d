"""mt_token_logprobs against a 64-bit implementation: vocabularies, types, ties, masks, rows without a distribution."""
import numpy as np
import pytest
import torch

from lm_util import code_of, init, logprob_bound, logprob_reference
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def run(logits, tokens, top):
    n = logits.shape[0]
    lp, ent = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ids, tlp = torch.full((n, top), 7, dtype=torch.int32, device="cuda"), torch.full((n, top), 7.0, device="cuda")
    mt.mt_token_logprobs(logits, torch.tensor(tokens, dtype=torch.int32, device="cuda"), lp, ent, ids, tlp)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in (lp, ent, ids, tlp)]


def check(logits, tokens, top):
    lp, ent, ids, tlp = run(logits, tokens, top)
    wl, we, wi, wt = logprob_reference(logits, tokens, top)
    assert np.array_equal(ids, wi)
    v = logits.shape[1]
    for got, want, size in ((lp, wl, 1), (tlp, wt, 1), (ent, we, 1)):
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
        ok = np.isfinite(want)
        x = np.abs(logits.double().cpu().numpy())
        big = np.where(np.isfinite(x), x, 0).max()
        if got is ent:                       # the mean of z is as exact as the sums, relative to its own size
            bound = logprob_bound(v, big) * (2 + 2 * np.abs(want[ok]))
        else:
            bound = logprob_bound(v, big + np.abs(want[ok]))
        err = np.abs(got.astype(np.float64)[ok] - want[ok])
        assert (err <= bound).all(), float(np.max(err / bound))


def rand(n, v, dtype=torch.float32, seed=0, pad=0, scale=3.0):
    init()
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (scale * torch.randn((n, v + pad), generator=g, device="cuda")).to(dtype)
    x[:, v:] = float("nan")
    return x[:, :v]


def toks(n, v, seed=0):
    return np.random.default_rng(seed).integers(0, v, n).tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1, 2, 31, 33, 255, 1000, 4096, 4097, 20001])
def test_vocabularies(dtype, v):
    for pad in (0, 3):
        check(rand(5, v, dtype, seed=v, pad=pad), toks(5, v), min(8, 32))


@pytest.mark.parametrize("top", [0, 1, 2, 5, 20, 31, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tops(top, dtype):
    check(rand(3, 5003, dtype, seed=top), toks(3, 5003), top)


@pytest.mark.parametrize("n,v", [(1, 200003), (2, 65536), (40, 33333), (400, 3001), (3000, 70)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows(n, v, dtype):
    check(rand(n, v, dtype, seed=n), toks(n, v), 10)


@pytest.mark.parametrize("v", [40, 3000, 50000])
def test_ties_go_to_the_lower_index(v):
    x = rand(6, v, torch.bfloat16)
    x[0] = 1.25                                         # all alike
    x[1] = torch.where(torch.arange(v, device="cuda") % 3 == 1, 2.0, -1.0).to(x.dtype)
    x[2] = x[2].round()
    x[3] = 0.0
    x[3, 1::2] = -0.0                                   # alike in value
    x[4] = torch.arange(v, device="cuda").to(x.dtype)   # rising, with long ties at the top
    x[5] = -torch.arange(v, device="cuda").to(x.dtype)
    check(x, toks(6, v), 32)
    check(x.float(), toks(6, v), 32)


@pytest.mark.parametrize("v", [40, 3000, 50000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks(v, dtype):
    x = rand(9, v, dtype, seed=1)
    low = torch.finfo(dtype).min
    inf = float("inf")
    x[0, 3:] = -inf                                     # three left
    x[1, :v - 1] = -inf                                 # the last one left
    x[2] = -inf                                         # none left
    x[3, 5] = float("nan")
    x[4, v - 1] = inf
    x[5, 4:] = low                                      # masked by the type's lowest value
    x[6] = low                                          # all of it
    x[7, ::2] = -inf
    x[8] = torch.where(torch.rand(v, device="cuda") < 0.01, x[8], torch.tensor(-inf, device="cuda", dtype=dtype))
    x[8, 0] = 0
    t = toks(9, v)
    t[0], t[1], t[5], t[7] = 1, 3, 10, 0
    lp, ent, ids, tlp = run(x, t, 20)
    keep = [0, 1, 2, 3, 4, 7, 8]
    check(x[keep], [t[i] for i in keep], 20)
    # rows with the lowest value: the mask's entries are ordinary logits of probability zero
    wl, we, wi, wt = logprob_reference(x[5:7], t[5:7], 20)
    assert np.array_equal(ids[5:7], wi)
    assert np.allclose(ent[5:7], we, rtol=1e-4, atol=1e-5)
    assert np.allclose(tlp[5:7].astype(np.float64), wt, rtol=1e-5) and np.allclose(lp[5:7].astype(np.float64), wl, rtol=1e-5)


def test_tokens_outside_the_vocabulary():
    x = rand(4, 300)
    lp, ent, ids, tlp = run(x, [-1, 300, 5, 2 ** 31 - 1], 3)
    assert np.isnan(lp[[0, 1, 3]]).all() and np.isfinite(lp[2]) and np.isfinite(ent).all() and (ids >= 0).all()
    assert mt.mt_get_async_status() == (0, -1)


def test_sorted_rows_and_repeated_blocks():
    """The largest values lie together: at the start, at the end, and all in one thread's share."""
    v = 40000
    x = rand(4, v, seed=3)
    x[0] = torch.sort(x[0], descending=True).values
    x[1] = torch.sort(x[1]).values
    x[2, 1000:1040] += 50
    x[3, ::1024] += 50
    check(x, toks(4, v), 32)
    check(x.to(torch.bfloat16), toks(4, v), 32)


def test_large_and_small_logits():
    x = rand(4, 3000, scale=1.0)
    x[0] *= 1e4
    x[1] += 1e5
    x[2] *= 1e-6
    x[3] = -1e30
    x[3, 17] = 1e30
    lp, ent, ids, tlp = run(x, [0, 1, 2, 17], 4)
    wl, we, wi, wt = logprob_reference(x, [0, 1, 2, 17], 4)
    assert np.array_equal(ids, wi)
    assert np.allclose(lp, wl, rtol=1e-5, atol=1e-4) and np.allclose(ent, we, rtol=1e-4, atol=1e-4)


def test_optional_outputs():
    x = rand(3, 500)
    t = toks(3, 500)
    want = run(x, t, 4)
    lp = torch.empty(3, device="cuda")
    mt.mt_token_logprobs(x, torch.tensor(t, dtype=torch.int32, device="cuda"), lp)
    assert np.array_equal(lp.cpu().numpy(), want[0])


def test_unaligned_rows():
    init()
    for dtype in (torch.bfloat16, torch.float32):
        buf = torch.randn(4 * 1001 + 7, device="cuda").to(dtype)
        for off in range(8 if dtype == torch.bfloat16 else 4):
            check(buf[off:off + 4 * 999].view(4, 999), toks(4, 999), 6)


def test_streams_and_repeats():
    a, b = rand(3, 60001, seed=1), rand(2, 30000, torch.bfloat16, seed=2)
    want = [run(a, toks(3, 60001), 9), run(b, toks(2, 30000), 9)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    args, outs = [], [[], []]
    for x in (a, b):
        args.append((x, torch.tensor(toks(*x.shape), dtype=torch.int32, device="cuda")))
    for j, x in enumerate((a, b)):
        n = x.shape[0]
        for _ in range(20):
            outs[j].append((torch.empty(n, device="cuda"), torch.empty(n, device="cuda"),
                            torch.empty((n, 9), dtype=torch.int32, device="cuda"), torch.empty((n, 9), device="cuda")))
    torch.cuda.synchronize()
    for i in range(20):
        for j in (0, 1):
            mt.mt_token_logprobs(*args[j], *outs[j][i], stream=streams[j])
    torch.cuda.synchronize()
    for w, rs in zip(want, outs):
        for r in rs:
            assert all(np.array_equal(x, y.cpu().numpy()) for x, y in zip(w, r))


def test_refusals():
    x = rand(3, 100)
    t = torch.zeros(3, dtype=torch.int32, device="cuda")
    lp = torch.empty(3, device="cuda")
    f = mt.mt_token_logprobs
    assert code_of(f, x.half(), t, lp) == 1
    assert code_of(f, x, t.long(), lp) == 1
    assert code_of(f, x, t, lp[:2]) == 1
    assert code_of(f, x, t, lp, None, torch.empty((3, 2), dtype=torch.int32, device="cuda"), None) == 1
    assert code_of(f, x, t, lp, None, torch.empty((3, 33), dtype=torch.int32, device="cuda"), torch.empty((3, 33), device="cuda")) == 4
    assert code_of(f, x[:, ::2], t, lp) == 1
    f(x[:0], t[:0], lp[:0])
    assert mt.mt_get_async_status() == (0, -1)
